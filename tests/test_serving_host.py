"""include/dar_serving.h without a GPU: the library exports what the header
declares, sizes workspaces and refuses bad arguments before anything is
enqueued. Device addresses are fake and never dereferenced, so the refusals
run only where no GPU is visible."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "dar_serving.h")

dar = pytest.importorskip("paper_2606_18587_amd", reason="libdar.so not built")

no_gpu = pytest.mark.skipif(torch.cuda.is_available(),
                            reason="fake device addresses are only used where no GPU exists")
FAKE, OTHER, MISALIGNED = 0x7f0000000000, 0x7e0000000000, 0x7f0000000008
BIG = 1 << 40


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(dar_[a-z_]+)\s*\(", text)))


def test_library_and_binding_hold_every_declared_name():
    names = declared()
    assert "dar_cache_evict" in names
    raw = ctypes.CDLL(dar.LIB_PATH)
    for n in names:
        assert hasattr(raw, n), n
        assert callable(getattr(dar, n)), n


def S(B=2, Hq=4, Hkv=2, d=64, dd=16, w=8, dtype=torch.bfloat16):
    return dar.make_shape(B, Hq, Hkv, d, dd, w, dtype)


def dense(cap=1000, n=900, **over):
    c = dar.DarCacheStruct(FAKE, FAKE, FAKE, OTHER, cap, n)
    for k, v in over.items():
        setattr(c, k, v)
    return c


def paged(**over):
    c = dar.DarPagedCacheStruct(FAKE, FAKE, FAKE, OTHER, FAKE, FAKE, 64, 16, 100)
    for k, v in over.items():
        setattr(c, k, v)
    return c


def test_evict_workspace():
    f = dar.dar_cache_evict_workspace_bytes
    rows = 4
    # per row an 8-byte result and two int lists of as many moves as can happen
    assert f(S(), 1000, 900) == rows * (8 + 8 * (1000 - 8 - 900))
    assert f(S(), 1000, 100) == rows * (8 + 8 * (100 + 7))
    assert f(S(), 1000, 992) == f(S(), 1000, 5000) == rows * 8
    assert f(S(w=0), 1000, 0) == rows * 8
    assert f(S(), 0, 1) == f(S(), 10, -1) == f(S(Hq=3), 10, 1) == 0


@no_gpu
@pytest.mark.parametrize("keep,fixed,sc,out,ws,ws_bytes,want", [
    (-1, 0, FAKE, FAKE, FAKE, BIG, dar.DAR_E_ARG),
    (100, -1, FAKE, FAKE, FAKE, BIG, dar.DAR_E_ARG),
    (100, 101, FAKE, FAKE, FAKE, BIG, dar.DAR_E_ARG),
    (100, 0, None, FAKE, FAKE, BIG, dar.DAR_E_ARG),
    (100, 0, FAKE, None, FAKE, BIG, dar.DAR_E_ARG),
    (100, 0, MISALIGNED, FAKE, FAKE, BIG, dar.DAR_E_ARG),
    (100, 0, FAKE, FAKE + 16, FAKE, BIG, dar.DAR_E_ARG),              # overlap in part
    (100, 0, FAKE + 2 * 2 * 1000 * 4 - 16, FAKE, FAKE, BIG, dar.DAR_E_ARG),
    (100, 0, FAKE, FAKE, None, BIG, dar.DAR_E_WORKSPACE),
    (100, 0, FAKE, FAKE, FAKE, 4 * (8 + 8 * 107) - 1, dar.DAR_E_WORKSPACE),
    (100, 0, FAKE, FAKE, MISALIGNED, BIG, dar.DAR_E_ARG),
])
def test_evict_refuses(keep, fixed, sc, out, ws, ws_bytes, want):
    s, c = S(), dense()
    assert dar.lib.dar_cache_evict(ctypes.byref(s), ctypes.byref(c), keep, fixed, sc, out, ws,
                                   ws_bytes, None) == want
    assert c.len == 900
    p = paged()
    if ws_bytes == BIG:
        assert dar.lib.dar_cache_evict_paged(ctypes.byref(s), ctypes.byref(p), keep, fixed, sc, out,
                                             ws, ws_bytes, None) == want


@no_gpu
def test_evict_refuses_caches():
    def call(c, s=None):
        return dar.lib.dar_cache_evict(ctypes.byref(s or S()), ctypes.byref(c) if c else None, 100, 0,
                                       FAKE, FAKE, FAKE, BIG, None)
    assert call(None) == dar.DAR_E_ARG
    for bad in (dict(v_lat=FAKE), dict(v_lat=None), dict(k_lat=MISALIGNED), dict(len=-1),
                dict(len=1001), dict(cap=0)):
        assert call(dense(**bad)) == dar.DAR_E_ARG, bad
    assert call(dense(), S(Hq=3)) == dar.DAR_E_ARG
    # nothing to evict and nothing to copy: no launch, no error
    assert call(dense(n=107)) == dar.DAR_OK
    assert call(dense(n=0)) == dar.DAR_OK

    def call_paged(p, s=None):
        return dar.lib.dar_cache_evict_paged(ctypes.byref(s or S()), ctypes.byref(p), 100, 0, FAKE,
                                             FAKE, FAKE, BIG, None)
    for bad in (dict(v_pool=FAKE), dict(k_pool=None), dict(page_size=48), dict(page_size=16),
                dict(max_blocks=0), dict(n_pages=0), dict(block_table=None), dict(lens=None),
                dict(lens=FAKE + 2), dict(max_blocks=1 << 26)):
        assert call_paged(paged(**bad)) == dar.DAR_E_ARG, bad


def al256(x):
    return (x + 255) // 256 * 256


def test_decode_workspaces():
    s = S()
    base = al256(dar.dar_decode_workspace_bytes(s, 1024))
    heads, dd = 8, 16
    tail = al256(heads * dd * 4) + al256(heads * 4)      # absorbed queries, denominators
    assert dar.dar_decode_scored_workspace_bytes(s, 1024) == base + tail
    assert dar.dar_decode_prefix_workspace_bytes(s, 1024, 0) == base + tail
    # the prefix's records {m, l, acc[d_down]}, a whole number of them a head
    with_prefix = dar.dar_decode_prefix_workspace_bytes(s, 1024, 512)
    assert base + tail + al256(heads * 18 * 4) <= with_prefix <= base + tail + al256(64 * heads * 18 * 4)
    for bad in ((S(Hq=3), 1024, 0), (S(Hq=12, Hkv=4), 1024, 0), (s, 0, 0), (s, 1024, -64), (s, 1024, 2048)):
        assert dar.dar_decode_prefix_workspace_bytes(*bad) == 0


def call_scored(s=None, c=None, q=FAKE, wd=FAKE, wu=None, o=FAKE, sc=FAKE, out=FAKE, ws=FAKE,
                ws_bytes=BIG):
    return dar.lib.dar_attn_decode_scored(ctypes.byref(s or S()), ctypes.byref(c or dense()), q, wd, wu,
                                          o, sc, out, ws, ws_bytes, None)


@no_gpu
@pytest.mark.parametrize("bad,want", [
    (dict(q=None), dar.DAR_E_ARG), (dict(wd=None), dar.DAR_E_ARG), (dict(o=MISALIGNED), dar.DAR_E_ARG),
    (dict(wu=MISALIGNED), dar.DAR_E_ARG), (dict(sc=None), dar.DAR_E_ARG), (dict(out=None), dar.DAR_E_ARG),
    (dict(sc=MISALIGNED), dar.DAR_E_ARG), (dict(out=FAKE + 64), dar.DAR_E_ARG),
    (dict(ws=None), dar.DAR_E_WORKSPACE), (dict(ws=MISALIGNED), dar.DAR_E_ARG),
    (dict(c=dense(n=0)), dar.DAR_E_ARG), (dict(c=dense(v_lat=FAKE)), dar.DAR_E_ARG),
    (dict(c=dense(k_win=None)), dar.DAR_E_ARG), (dict(s=S(Hq=3)), dar.DAR_E_ARG),
    (dict(s=S(Hq=6)), dar.DAR_E_UNSUPPORTED), (dict(s=S(d=300, dd=16)), dar.DAR_E_UNSUPPORTED),
])
def test_scored_refuses(bad, want):
    assert call_scored(**bad) == want


@no_gpu
def test_scored_refuses_short_workspace():
    need = dar.dar_decode_scored_workspace_bytes(S(), 1000)
    assert call_scored(ws_bytes=need - 1) == dar.DAR_E_WORKSPACE


@no_gpu
@pytest.mark.parametrize("bad,want", [
    (dict(n=-64), dar.DAR_E_ARG), (dict(n=32), dar.DAR_E_ARG), (dict(n=1088), dar.DAR_E_ARG),
    (dict(n=64, blocks=None), dar.DAR_E_ARG), (dict(n=64, blocks=FAKE + 2), dar.DAR_E_ARG),
    (dict(q=None), dar.DAR_E_ARG), (dict(o=None), dar.DAR_E_ARG), (dict(wu=MISALIGNED), dar.DAR_E_ARG),
    (dict(c=paged(page_size=48)), dar.DAR_E_ARG), (dict(c=paged(lens=None)), dar.DAR_E_ARG),
    (dict(s=S(dtype=torch.float32)), dar.DAR_E_UNSUPPORTED), (dict(s=S(dd=24)), dar.DAR_E_UNSUPPORTED),
    (dict(s=S(d=80)), dar.DAR_E_UNSUPPORTED), (dict(s=S(Hq=32)), dar.DAR_E_UNSUPPORTED),
    (dict(ws=None), dar.DAR_E_WORKSPACE), (dict(ws_bytes=1000), dar.DAR_E_WORKSPACE),
    (dict(ws=MISALIGNED), dar.DAR_E_ARG),
])
def test_prefix_refuses(bad, want):
    a = dict(s=S(), c=paged(), n=512, blocks=FAKE, q=FAKE, wd=FAKE, wu=None, o=FAKE, ws=FAKE, ws_bytes=BIG)
    a.update(bad)
    head = (ctypes.byref(a["s"]), ctypes.byref(a["c"]), a["n"], a["blocks"], a["q"], a["wd"], a["wu"], a["o"])
    assert dar.lib.dar_attn_decode_paged_prefix(*head, a["ws"], a["ws_bytes"], None) == want
    assert dar.lib.dar_attn_decode_paged_scored(*head, FAKE, FAKE, a["ws"], a["ws_bytes"], None) == want


@no_gpu
def test_paged_scored_refuses_scores():
    for sc, out in ((None, FAKE), (FAKE, None), (FAKE, MISALIGNED), (FAKE, FAKE + 16)):
        assert dar.lib.dar_attn_decode_paged_scored(
            ctypes.byref(S()), ctypes.byref(paged()), 0, None, FAKE, FAKE, None, FAKE, sc, out, FAKE, BIG,
            None) == dar.DAR_E_ARG


@no_gpu
def test_refuses_what_token_numbers_and_grids_do_not_hold():
    long = (1 << 30) + 64
    assert call_scored(c=dense(cap=long)) == dar.DAR_E_UNSUPPORTED
    wide = S(B=40000)
    assert call_scored(s=wide) == dar.DAR_E_UNSUPPORTED
    for s, p in ((S(), paged(max_blocks=long // 64)), (wide, paged())):
        head = (ctypes.byref(s), ctypes.byref(p), 64, FAKE, FAKE, FAKE, None, FAKE)
        assert dar.lib.dar_attn_decode_paged_prefix(*head, FAKE, BIG, None) == dar.DAR_E_UNSUPPORTED
        assert dar.lib.dar_attn_decode_paged_scored(*head, FAKE, FAKE, FAKE, BIG,
                                                    None) == dar.DAR_E_UNSUPPORTED
        assert dar.lib.dar_cache_evict_paged(ctypes.byref(s), ctypes.byref(p), 100, 0, FAKE, FAKE, FAKE,
                                             BIG, None) == dar.DAR_E_UNSUPPORTED
    for s, c in ((S(), dense(cap=long)), (wide, dense())):
        assert dar.lib.dar_cache_evict(ctypes.byref(s), ctypes.byref(c), 100, 0, FAKE, FAKE, FAKE, BIG,
                                       None) == dar.DAR_E_UNSUPPORTED


@no_gpu
def test_decodes_refuse_what_32_bit_offsets_do_not_hold():
    """Latents are read through 32-bit byte offsets: from a head's first row in the
    dense decodes, whose capacities stay far below them, and from a page's."""
    for dtype in (torch.bfloat16, torch.float32):
        for dd in (16, 32):
            for cap in (1 << 21, 1 << 26, 1 << 30):
                assert call_scored(S(dd=dd, dtype=dtype), dense(cap=cap, n=cap)) == dar.DAR_E_UNSUPPORTED

    def calls(dd, page):
        s, c = S(dd=dd), paged(page_size=page, max_blocks=1)
        head = (ctypes.byref(s), ctypes.byref(c))
        tail = (FAKE, FAKE, None, FAKE)
        return (dar.lib.dar_attn_decode_paged_prefix(*head, 0, None, *tail, FAKE, 0, None),
                dar.lib.dar_attn_decode_paged_scored(*head, 0, None, *tail, FAKE, FAKE, FAKE, 0, None),
                dar.lib.dar_attn_decode_paged(*head, *tail, FAKE, 0, None))
    for dd in (16, 32):
        fits = (1 << 31) // (2 * dd)
        assert calls(dd, 2 * fits) == (dar.DAR_E_UNSUPPORTED,) * 3
        assert calls(dd, fits) == (dar.DAR_E_WORKSPACE,) * 3


def test_binding_refuses():
    """Shapes, types and devices are checked before the library is called."""
    c = dar.DarCache(2, 2, 64, 16, 8, 100, torch.bfloat16, device="cpu")
    good = torch.zeros(2, 2, 100)
    for bad in (torch.zeros(2, 2, 99), good.double(), torch.zeros(2, 200), good.to("meta")):
        with pytest.raises(ValueError):
            dar._check_scores(c, bad, None)
        with pytest.raises(ValueError):
            dar._check_scores(c, good, bad)
    q, wd = torch.zeros(2, 4, 64).bfloat16(), torch.zeros(2, 64, 16).bfloat16()
    dar._check_step(c, q, wd, None, None)
    for args in ((q[:1], wd, None, None), (q.float(), wd, None, None), (q, wd.float(), None, None),
                 (q, wd[:, :, :8], None, None), (q, wd, wd, None), (q, wd, None, q[:, :2]),
                 (q.to("meta"), wd, None, None)):
        with pytest.raises(ValueError):
            dar._check_step(c, *args)
    p = dar.DarPagedCache(2, 2, 64, 16, 8, 64, 4, 8, torch.bfloat16, device="cpu")
    assert dar._prefix(p, None) == 0 and dar._prefix(p, torch.zeros(3, dtype=torch.int32)) == 192
    for bad in (torch.zeros(3), torch.zeros(1, 3, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)):
        with pytest.raises(ValueError):
            dar._prefix(p, bad)


@no_gpu
def test_binding_refuses_numbers_that_are_no_c_int(monkeypatch):
    """Not taken modulo 2^32: n_keep of 2^32 ("keep everything") is not 0, and n_fixed
    and the workspace sizes' arguments neither."""
    called = []
    monkeypatch.setattr(dar, "_on", lambda cache, stream: dar._HERE)
    monkeypatch.setattr(dar, "_stream", lambda stream: called.append(stream))
    c = dar.DarCache(2, 2, 64, 16, 8, 100, torch.bfloat16, device="cpu")
    c.struct.len = 90
    p = dar.DarPagedCache(2, 2, 64, 16, 8, 64, 4, 8, torch.bfloat16, device="cpu")
    for f, cache, cap in ((dar.dar_cache_evict, c, 100), (dar.dar_cache_evict_paged, p, 256)):
        for keep, fixed in ((1 << 32, 0), (1 << 31, 0), (50, 1 << 32), (-1 << 32, 0)):
            with pytest.raises(ValueError):
                f(cache, torch.zeros(2, 2, cap), keep, n_fixed=fixed)
    with pytest.raises(ValueError):
        dar.dar_cache_evict_workspace_bytes(S(), 1000, 1 << 32)
    with pytest.raises(ValueError):
        dar.dar_decode_prefix_workspace_bytes(S(), 1 << 33, 0)
    with pytest.raises(ValueError):
        dar._prefix(p, torch.zeros(1, dtype=torch.int32).expand(1 << 26))
    assert not called and c.len == 90
