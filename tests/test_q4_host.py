"""include/dar_q4.h without a GPU: the library exports what the header declares,
sizes workspaces and refuses bad arguments before anything is enqueued. Device
addresses are fake and never dereferenced, so the refusals run only where no GPU
is visible. The reference of the GPU tests is pinned here, too."""
import contextlib
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from tests import q4_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "dar_q4.h")

dar = pytest.importorskip("paper_2606_18587_amd", reason="libdar.so not built")

no_gpu = pytest.mark.skipif(torch.cuda.is_available(),
                            reason="fake device addresses are only used where no GPU exists")
FAKE, OTHER, MISALIGNED = 0x7f0000000000, 0x7e0000000000, 0x7f0000000008
BIG = 1 << 40
LONG = (1 << 30) + 64
BF = torch.bfloat16


def test_reference_on_known_values():
    """The format's rules on values worked out by hand."""
    x = np.array([[7.0, 6.5, 5.0, -5.0, 4.9, 2.5, 1.25, 0.75, 0.25, -0.25, 0.0, -3.5]])
    codes, exps = ref.quantise(x)
    assert exps.tolist() == [[127]]
    assert ref.values(codes, exps, 12).tolist() == [[6, 6, 4, -4, 4, 2, 1, 1, 0, 0, 0, -4]]
    assert codes.shape == (1, 8) and (codes[:, 6:] == 0).all()
    _, exps = ref.quantise(np.array([[7.0625, 0.0], [14.0, 1.0], [0.0, 0.0], [np.inf, 1.0], [3e38, 0], [1e-45, 0]]))
    assert exps[:, 0].tolist() == [128, 128, 3, 255, 252, 3]
    wide = np.zeros((1, 33))
    wide[0, 32], wide[0, 0] = 6.0, np.nan
    codes, exps = ref.quantise(wide)
    assert exps.tolist() == [[255, 127]] and codes.shape == (1, 20)
    got = ref.values(codes, exps, 33)[0]
    assert np.isnan(got[:32]).all() and got[32] == 6


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(dar_[a-z0-9_]+)\s*\(", text)))


def test_library_and_binding_hold_every_declared_name():
    names = declared()
    assert len(names) == 9 and "dar_attn_decode_paged_q4" in names
    raw = ctypes.CDLL(dar.LIB_PATH)
    for n in names:
        assert hasattr(raw, n), n
        assert callable(getattr(dar, n)), n


def S(B=2, Hq=4, Hkv=2, d=64, dd=16, w=8, dtype=BF):
    return dar.make_shape(B, Hq, Hkv, d, dd, w, dtype)


def made(cls, names, more, over):
    c = cls(**dict({n: FAKE for n in names}, **more))
    for k, v in over.items():
        setattr(c, k, v)
    return c


Q4_ARRAYS = ("k_win", "v_win", "k_codes", "v_codes", "k_exp", "v_exp")


def q4(**over):
    return made(dar.DarCacheQ4Struct, Q4_ARRAYS, dict(cap=1024, len=900), over)


def q4_paged(**over):
    return made(dar.DarPagedCacheQ4Struct, Q4_ARRAYS + ("block_table", "lens"),
                dict(page_size=64, max_blocks=16, n_pages=100), over)


def dense(**over):
    return made(dar.DarCacheStruct, ("k_win", "v_win", "k_lat"), dict(v_lat=OTHER, cap=1000, len=900), over)


def paged(**over):
    return made(dar.DarPagedCacheStruct, ("k_win", "v_win", "k_pool", "block_table", "lens"),
                dict(v_pool=OTHER, page_size=64, max_blocks=16, n_pages=100), over)


ref_ = ctypes.byref
BAD_SHAPES = [(dict(Hq=3), dar.DAR_E_ARG), (dict(dd=65), dar.DAR_E_ARG), (dict(d=300), dar.DAR_E_UNSUPPORTED),
              (dict(B=40000), dar.DAR_E_UNSUPPORTED)]
BAD_ARRAYS = [dict(zip((n,), (v,))) for n in Q4_ARRAYS for v in (None, MISALIGNED)]
BAD_PAGES = [dict(page_size=48), dict(page_size=16), dict(max_blocks=0), dict(n_pages=0), dict(block_table=None),
             dict(lens=None), dict(lens=FAKE + 2), dict(max_blocks=1 << 26)]


def test_workspace():
    f = dar.dar_decode_q4_workspace_bytes
    assert f(S(), 1024) == f(S(), 64) > 0 and f(S(), 1024) % 256 == 0
    assert f(S(Hq=16), 1024) > f(S(Hq=8), 1024)
    for bad in ((S(Hq=3), 64), (S(), 0), (S(), -64), (S(), LONG), (S(d=300), 64)):
        assert f(*bad) == 0


def append(s=None, c=None, n=1, k=FAKE, v=FAKE, wd=FAKE):
    return dar.lib.dar_cache_append_q4(ref_(s or S()), ref_(c) if c else None, k, v, n, wd, None)


@no_gpu
def test_append_refuses():
    for s, want in BAD_SHAPES:
        assert append(S(**s), q4()) == want, s
    assert append(c=None) == dar.DAR_E_ARG
    for bad in BAD_ARRAYS + [dict(cap=1000), dict(cap=0), dict(len=-1), dict(len=1025)]:
        assert append(c=q4(**bad)) == dar.DAR_E_ARG, bad
    assert append(c=q4(cap=LONG)) == dar.DAR_E_UNSUPPORTED
    for bad in (dict(n=0), dict(n=-1), dict(k=None), dict(v=MISALIGNED), dict(wd=None)):
        assert append(c=q4(), **bad) == dar.DAR_E_ARG, bad
    c = q4()
    assert append(c=c, n=125) == dar.DAR_E_CAPACITY and append(c=c, n=2 ** 31 - 1) == dar.DAR_E_CAPACITY
    assert c.len == 900

    def step(s=None, c=None, k=FAKE, v=FAKE, wd=FAKE):
        return dar.lib.dar_cache_append_paged_q4(ref_(s or S()), ref_(c or q4_paged()), k, v, wd, None)
    for s, want in BAD_SHAPES:
        assert step(S(**s)) == want, s
    for bad in BAD_ARRAYS + BAD_PAGES:
        assert step(c=q4_paged(**bad)) == dar.DAR_E_ARG, bad
    assert step(c=q4_paged(max_blocks=LONG // 64)) == dar.DAR_E_UNSUPPORTED
    for bad in (dict(k=None), dict(v=MISALIGNED), dict(wd=None)):
        assert step(**bad) == dar.DAR_E_ARG, bad


@no_gpu
def test_conversions_refuse():
    codes = [b for b in BAD_ARRAYS if "win" not in next(iter(b))]

    def pack(s=None, src=None, first=0, dst=None):
        return dar.lib.dar_cache_pack_q4(ref_(s or S()), ref_(src or dense()), first, ref_(dst or q4()), None)

    def unpack(s=None, src=None, first=0, dst=None):
        return dar.lib.dar_cache_unpack_q4(ref_(s or S()), ref_(src or q4()), first, ref_(dst or dense()), None)
    for f in (pack, unpack):
        for s, want in BAD_SHAPES:
            assert f(S(**s)) == want, s
        assert f(first=-1) == dar.DAR_E_ARG
    lat = [dict(k_lat=None), dict(v_lat=MISALIGNED), dict(v_lat=FAKE), dict(cap=0)]
    for bad in lat + [dict(len=-1), dict(len=1001)]:
        assert pack(src=dense(**bad)) == dar.DAR_E_ARG, bad
    for bad in lat:
        assert unpack(dst=dense(**bad)) == dar.DAR_E_ARG, bad
    for bad in codes + [dict(cap=1000)]:
        assert pack(dst=q4(**bad)) == unpack(src=q4(**bad)) == dar.DAR_E_ARG, bad
    assert unpack(src=q4(len=1025)) == dar.DAR_E_ARG
    assert pack(dst=q4(cap=LONG)) == pack(src=dense(cap=LONG)) == dar.DAR_E_UNSUPPORTED
    assert pack(dst=q4(cap=832)) == dar.DAR_E_CAPACITY and unpack(dst=dense(cap=899)) == dar.DAR_E_CAPACITY
    # nothing to convert: no launch, no error, and the length follows
    d, c = dense(len=0), q4()
    assert pack(src=dense(len=8), dst=c) == dar.DAR_OK and c.len == 8
    assert pack(first=892, dst=c) == dar.DAR_OK and c.len == 900
    assert unpack(src=q4(len=5), dst=d) == dar.DAR_OK and d.len == 5
    d.len = -77  # (what the destination held does not matter)
    assert unpack(src=q4(len=5), dst=d) == dar.DAR_OK and d.len == 5
    assert pack(dst=q4(k_win=None, v_win=None), src=dense(len=3, k_win=None)) == dar.DAR_OK

    def pack_paged(s=None, src=None, first=None, dst=None):
        return dar.lib.dar_cache_pack_paged_q4(ref_(s or S()), ref_(src or paged()), first, ref_(dst or q4_paged()), None)

    def unpack_paged(s=None, src=None, first=None, dst=None):
        return dar.lib.dar_cache_unpack_paged_q4(ref_(s or S()), ref_(src or q4_paged()), first, ref_(dst or paged()), None)
    for f in (pack_paged, unpack_paged):
        for s, want in BAD_SHAPES:
            assert f(S(**s)) == want, s
        assert f(first=FAKE + 2) == dar.DAR_E_ARG
    for bad in [dict(k_pool=None), dict(v_pool=FAKE), dict(v_pool=MISALIGNED)] + BAD_PAGES:
        assert pack_paged(src=paged(**bad)) == unpack_paged(dst=paged(**bad)) == dar.DAR_E_ARG, bad
    for bad in codes + BAD_PAGES:
        assert pack_paged(dst=q4_paged(**bad)) == unpack_paged(src=q4_paged(**bad)) == dar.DAR_E_ARG, bad


@no_gpu
def test_paged_conversions_refuse_lengths_that_others_read():
    """The destination's lengths are written by the launch that reads first and the
    source's lengths: they share no element, unless both lengths are one array."""
    B, at = 5, OTHER + 4096

    def pack(src, first, dst):
        return dar.lib.dar_cache_pack_paged_q4(ref_(S(B=B)), ref_(paged(lens=src)), first, ref_(q4_paged(lens=dst)), None)

    def unpack(src, first, dst):
        return dar.lib.dar_cache_unpack_paged_q4(ref_(S(B=B)), ref_(q4_paged(lens=src)), first, ref_(paged(lens=dst)), None)
    for f in (pack, unpack):
        for k in (4 * B - 4, 4, 0, -4, 4 - 4 * B):
            assert f(FAKE, at + k, at) == dar.DAR_E_ARG, k
            if k:
                assert f(at + k, None, at) == dar.DAR_E_ARG, k
        # (these go on to the launch, which has no device here)
        for args in ((FAKE, at + 4 * B, at), (FAKE, at - 4 * B, at), (at + 4 * B, None, at), (at, at, at), (at, at + 4, at)):
            assert f(*args) == dar.DAR_E_HIP, args


@no_gpu
def test_decode_refuses():
    def dec(s=None, c=None, q=FAKE, wd=FAKE, wu=None, o=FAKE, ws=FAKE, wsb=BIG):
        return dar.lib.dar_attn_decode_q4(ref_(s or S()), ref_(c or q4()), q, wd, wu, o, ws, wsb, None)

    def dec_paged(s=None, c=None, q=FAKE, wd=FAKE, wu=None, o=FAKE, ws=FAKE, wsb=BIG):
        return dar.lib.dar_attn_decode_paged_q4(ref_(s or S()), ref_(c or q4_paged()), q, wd, wu, o, ws, wsb, None)
    need = dar.dar_decode_q4_workspace_bytes(S(), 1024)
    for f in (dec, dec_paged):
        for s, want in BAD_SHAPES:
            assert f(S(**s)) == want, s
        for bad in (dict(q=None), dict(wd=MISALIGNED), dict(wu=MISALIGNED), dict(o=None), dict(ws=MISALIGNED)):
            assert f(**bad) == dar.DAR_E_ARG, bad
        assert f(ws=None) == f(wsb=need - 1) == dar.DAR_E_WORKSPACE
    for bad in BAD_ARRAYS + [dict(cap=1000), dict(len=0), dict(len=1025)]:
        assert dec(c=q4(**bad)) == dar.DAR_E_ARG, bad
    assert dec(c=q4(cap=LONG, len=5)) == dar.DAR_E_UNSUPPORTED
    for bad in BAD_ARRAYS + BAD_PAGES:
        assert dec_paged(c=q4_paged(**bad)) == dar.DAR_E_ARG, bad
    assert dec_paged(c=q4_paged(max_blocks=LONG // 64)) == dar.DAR_E_UNSUPPORTED
    # more work, all sequences full, than is numbered in 32 bits
    assert dec_paged(S(B=400, Hq=8, Hkv=8), q4_paged(max_blocks=1 << 24)) == dar.DAR_E_UNSUPPORTED


@no_gpu
def test_limit_of_the_batch():
    """B * Hkv is what the caches are limited by, up to 65535; a decode takes 2^20 query
    heads."""
    many = dict(B=2048, Hq=64, Hkv=8)                      # 16384 KV heads, 131072 query heads
    edge = [(dict(B=65535, Hq=1, Hkv=1), True), (dict(B=65536, Hq=1, Hkv=1), False), (dict(B=13107, Hq=20, Hkv=5), True),
            (dict(B=21846, Hq=3, Hkv=3), False), (many, True)]
    for s, fits in edge:
        s = S(**s)
        assert append(s, q4(), n=125) == (dar.DAR_E_CAPACITY if fits else dar.DAR_E_UNSUPPORTED)
        for f, a, b in ((dar.lib.dar_cache_pack_q4, dense(len=8), q4()), (dar.lib.dar_cache_unpack_q4, q4(len=8), dense())):
            assert f(ref_(s), ref_(a), 0, ref_(b), None) == (dar.DAR_OK if fits else dar.DAR_E_UNSUPPORTED)
        for f, a, b in ((dar.lib.dar_cache_pack_paged_q4, paged(), q4_paged(k_codes=None)),
                        (dar.lib.dar_cache_unpack_paged_q4, q4_paged(k_codes=None), paged())):
            assert f(ref_(s), ref_(a), None, ref_(b), None) == (dar.DAR_E_ARG if fits else dar.DAR_E_UNSUPPORTED)
        assert dar.lib.dar_cache_append_paged_q4(ref_(s), ref_(q4_paged()), None, FAKE, FAKE, None) == (
            dar.DAR_E_ARG if fits else dar.DAR_E_UNSUPPORTED)
    def decode(s, want):
        for f, c in ((dar.lib.dar_attn_decode_q4, q4()), (dar.lib.dar_attn_decode_paged_q4, q4_paged())):
            assert f(ref_(s), ref_(c), FAKE, FAKE, None, FAKE, None, 0, None) == want
        assert (dar.dar_decode_q4_workspace_bytes(s, 1024) > 0) == (want == dar.DAR_E_WORKSPACE)
    for s, fits in edge + [(dict(B=1 << 10, Hq=1 << 10, Hkv=4), True), (dict(B=1 << 10, Hq=1028, Hkv=4), False),
                           (dict(B=1, Hq=1 << 20, Hkv=1), True), (dict(B=2, Hq=2 ** 31 - 1, Hkv=1), False)]:
        decode(S(**s), dar.DAR_E_WORKSPACE if fits else dar.DAR_E_UNSUPPORTED)


class Launches:
    """The library with every entry point that would launch replaced."""

    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return getattr(self.real, name)

        def call(*args):
            self.calls.append((name, args[-1]))
            return dar.DAR_OK
        return call


class FakeStream:
    cuda_stream = 0x1234
    device = torch.device("cpu")


def caches():
    shape = (2, 2, 64, 16, 8)
    a = dar.DarCacheQ4(*shape, 100, BF, device="cpu"), dar.DarCache(*shape, 100, BF, device="cpu")
    b = (dar.DarPagedCacheQ4(*shape, 64, 4, 8, BF, device="cpu"), dar.DarPagedCache(*shape, 64, 4, 8, BF, device="cpu"))
    return a + b


def test_caches():
    c, plain, p, pp = caches()
    assert c.cap == c.struct.cap == 128 and c.len == 0
    assert c.k_codes.shape == (2, 2, 128, 8) and c.v_exp.shape == (2, 2, 128, 1)
    assert p.k_codes.shape == (8, 2, 64, 8) and p.cap == 256 and p.overflowed() == []
    wide = dar.DarCacheQ4(1, 1, 64, 33, 0, 64, BF, device="cpu")
    assert wide.k_codes.shape == (1, 1, 64, 20) and wide.k_exp.shape == (1, 1, 64, 2)
    assert c.share_ring(plain) is c and c.struct.k_win == plain.k_win.data_ptr()
    assert p.share_ring(pp).lens is pp.lens
    other = dar.DarCache(2, 2, 64, 16, 9, 100, BF, device="cpu")
    with pytest.raises(ValueError):
        c.share_ring(other)
    with pytest.raises(ValueError):
        dar.DarCacheQ4(1, 1, 64, 16, 8, 1 << 33, BF, device="cpu")


def test_binding_refuses(monkeypatch):
    """Shapes, types, devices and caches that do not match are refused before the
    library is called."""
    launches = Launches(dar.lib)
    monkeypatch.setattr(dar, "lib", launches)
    monkeypatch.setattr(dar, "_on", lambda cache, stream: dar._HERE)
    monkeypatch.setattr(dar, "_stream", lambda stream: 0)
    c, plain, p, pp = caches()
    k, wd = torch.zeros(2, 2, 3, 64).to(BF), torch.zeros(2, 64, 16).to(BF)
    dar.dar_cache_append_q4(c, k, k, wd)
    dar.dar_cache_append_paged_q4(p, k[:, :, 0].contiguous(), k[:, :, 0].contiguous(), wd)
    n = len(launches.calls)
    for args in ((k[:1], k, wd), (k, k[:, :, :2], wd), (k.float(), k.float(), wd), (k, k, wd.float()),
                 (k, k, wd[:, :, :8]), (k.to("meta"), k, wd), (k[:, :, 0], k[:, :, 0], wd),
                 (k[..., ::2], k[..., ::2], wd), (k.transpose(0, 1), k, wd)):
        with pytest.raises(ValueError):
            dar.dar_cache_append_q4(c, *args)
        with pytest.raises(ValueError):
            dar.dar_cache_append_paged_q4(p, *args)
    for f, a, b in ((dar.dar_cache_pack_q4, plain, c), (dar.dar_cache_unpack_q4, c, plain)):
        for bad in (1 << 31, 1 << 32, -1 << 32):
            with pytest.raises(ValueError):
                f(a, b, first=bad)
        with pytest.raises(ValueError):
            f(a, dar.DarCache(2, 2, 64, 16, 8, 100, torch.float32, device="cpu"))
        with pytest.raises(ValueError):
            f(a, dar.DarCache(1, 2, 64, 16, 8, 100, BF, device="cpu"))
    with pytest.raises(ValueError):
        dar.dar_cache_pack_q4(dar.DarCache(2, 2, 64, 16, 8, 100, BF, device="cpu", shared=True), c)
    for f, a, b in ((dar.dar_cache_pack_paged_q4, pp, p), (dar.dar_cache_unpack_paged_q4, p, pp)):
        for bad in (torch.zeros(2), torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int64),
                    torch.zeros(2, dtype=torch.int32, device="meta")):
            with pytest.raises(ValueError):
                f(a, b, first=bad)
    q = torch.zeros(2, 4, 64).to(BF)
    for f, cache in ((dar.dar_attn_decode_q4, c), (dar.dar_attn_decode_paged_q4, p)):
        for args in ((q[:1], wd), (q.float(), wd), (q, wd.float()), (q, wd, wd), (q.to("meta"), wd)):
            with pytest.raises(ValueError):
                f(cache, *args)
    for a, bad in (("lens", torch.zeros(2, dtype=torch.int64)), ("block_table", torch.zeros(2, 3, dtype=torch.int32)),
                   ("lens", torch.zeros(4, dtype=torch.int32)[::2])):
        broken = caches()[2]
        setattr(broken, a, bad)
        with pytest.raises(ValueError):
            dar.dar_attn_decode_paged_q4(broken, q, wd)
    with pytest.raises(ValueError):
        dar.dar_decode_q4_workspace_bytes(S(), 1 << 32)
    assert len(launches.calls) == n


def test_calls_and_allocations_go_to_the_stream(monkeypatch):
    current, taken = [], []

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    def watched(real):
        def make(*args, **kw):
            taken.append(current[-1] if current else None)
            return real(*args, **kw)
        return make
    c, plain, p, pp = caches()
    c.struct.len = 60
    k, wd, q = torch.zeros(2, 2, 1, 64).to(BF), torch.zeros(2, 64, 16).to(BF), torch.zeros(2, 4, 64).to(BF)
    one = torch.zeros(2, 2, 64).to(BF)
    launches, s = Launches(dar.lib), FakeStream()
    monkeypatch.setattr(dar, "lib", launches)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", watched(torch.empty))
    monkeypatch.setattr(torch, "empty_like", watched(torch.empty_like))
    calls = [lambda s: dar.dar_cache_append_q4(c, k, k, wd, stream=s),
             lambda s: dar.dar_cache_append_paged_q4(p, one, one, wd, stream=s),
             lambda s: dar.dar_cache_pack_q4(plain, c, stream=s), lambda s: dar.dar_cache_unpack_q4(c, plain, stream=s),
             lambda s: dar.dar_cache_pack_paged_q4(pp, p, stream=s),
             lambda s: dar.dar_cache_unpack_paged_q4(p, pp, stream=s),
             lambda s: dar.dar_attn_decode_q4(c, q, wd, stream=s),
             lambda s: dar.dar_attn_decode_paged_q4(p, q, wd, stream=s)]
    for f in calls:
        f(s)
    assert len(launches.calls) == len(calls) and all(x == s.cuda_stream for _, x in launches.calls)
    assert len(taken) == 4 and all(x is s for x in taken)
    other = FakeStream()
    other.device = torch.device("cuda", 1)
    for f in calls:
        with pytest.raises(ValueError, match="stream"):
            f(other)
