"""The 4-bit cache on the GPU against its definitions in fp64: packing, reading
back, appends, decode steps, dense and paged; then the operators together, under
graphs and on other streams."""
import numpy as np
import pytest
import torch

from tests import q4_ref as ref

pytestmark = pytest.mark.gpu

dar = pytest.importorskip("paper_2606_18587_amd")

BF, F32 = torch.bfloat16, torch.float32


def f64(x):
    return x.detach().double().cpu().numpy()


def randn(g, *shape, dtype=BF, std=1.0):
    return (torch.randn(*shape, generator=g) * std).to(dtype).cuda()


def gen(seed):
    return torch.Generator().manual_seed(seed)


# --- packing and reading back ---------------------------------------------------

def special_rows(dd, dtype):
    """Rows where the format's rules meet: zeros, ties, saturation, the smallest and
    largest scales, infinities and NaN."""
    r = torch.arange(dd, dtype=torch.float64)
    rows = [torch.zeros(dd), -torch.zeros(dd), 0.25 * (r % 29), -0.25 * (r % 25), (r % 8) - 3.5,
            7.0 - 0.0625 * r, 7.0625 * (r == dd - 1), 6.0 * (r == 0) + 6.9375 * (r == dd // 2),
            3.0e38 * ((r % 3) - 1), 1.0e-38 * (r + 1), 2.0 ** -126 * (r % 5), 2.0 ** -130 * (r + 1),
            2.0 ** 120 * (r + 1), 1e-30 * r - 3e-30, torch.full((dd,), float("inf")),
            torch.where(r == dd - 1, float("nan"), 1.0), torch.where(r == 0, -float("inf"), r),
            2.0 ** (r % 60 - 30)]
    return torch.stack([x.double() for x in rows]).to(dtype)


def check_rows(codes, exps, x, dd):
    """Codes and scale bytes against the reference, byte by byte."""
    c, e = ref.quantise(f64(x).reshape(-1, dd))
    assert np.array_equal(exps.cpu().numpy().reshape(e.shape), e)
    assert np.array_equal(codes.cpu().numpy().reshape(c.shape), c)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dd,n,first", [(16, 1, 0), (16, 700, 0), (16, 513, 130), (32, 65, 0), (32, 259, 7),
                                        (1, 40, 0), (7, 70, 3), (20, 300, 0), (33, 70, 0), (64, 50, 1), (100, 41, 0)])
def test_pack_and_unpack(dtype, dd, n, first):
    B, Hkv, d, w, cap = 2, 3, 128, 5, n + 40
    g = gen(n + dd)
    src = dar.DarCache(B, Hkv, d, dd, w, cap, dtype)
    q4 = dar.DarCacheQ4(B, Hkv, d, dd, w, cap, dtype)
    back = dar.DarCache(B, Hkv, d, dd, w, cap + 3, dtype)
    for lat in (src.k_lat, src.v_lat):
        lat.copy_(randn(g, *lat.shape, dtype=dtype) * torch.exp2(torch.randint(-20, 20, (B, Hkv, cap, 1), generator=g)).cuda())
        rows = special_rows(dd, dtype).cuda()
        at = torch.randperm(n, generator=g)[:min(n, len(rows))]
        lat[0, 1, at.cuda()] = rows[:len(at)]
    src.struct.len = n + w
    for t in (q4.k_codes, q4.v_codes, q4.k_exp, q4.v_exp):
        t.fill_(0xA5)
    for t in (back.k_lat, back.v_lat):
        t.fill_(17.0)
    assert dar.dar_cache_pack_q4(src, q4, first=first) is q4 and q4.len == n + w
    assert dar.dar_cache_unpack_q4(q4, back, first=first) is back and back.len == n + w
    for lat, codes, exps, out in ((src.k_lat, q4.k_codes, q4.k_exp, back.k_lat),
                                  (src.v_lat, q4.v_codes, q4.v_exp, back.v_lat)):
        check_rows(codes[:, :, first:n], exps[:, :, first:n], lat[:, :, first:n], dd)
        for a in (codes, exps):                     # rows not asked for stay as they were
            assert (a[:, :, :first] == 0xA5).all() and (a[:, :, n:] == 0xA5).all()
        want = ref.values(codes.cpu().numpy()[:, :, first:n].reshape(-1, codes.shape[3]),
                          exps.cpu().numpy()[:, :, first:n].reshape(-1, exps.shape[3]), dd)
        assert np.array_equal(f64(out[:, :, first:n]).reshape(-1, dd), want, equal_nan=True)
        assert (out[:, :, :first] == 17).all() and (out[:, :, n:] == 17).all()


@pytest.mark.parametrize("dtype,dd", [(BF, 16), (BF, 32), (F32, 20)])
def test_nothing_to_convert(dtype, dd):
    """Windows that hold everything, and a first at or past the end."""
    src = dar.DarCache(1, 2, 64, dd, 8, 100, dtype)
    q4 = dar.DarCacheQ4(1, 2, 64, dd, 8, 100, dtype)
    q4.k_codes.fill_(3)
    for n, first in ((0, 0), (1, 0), (8, 0), (50, 42), (50, 1000)):
        src.struct.len = n
        dar.dar_cache_pack_q4(src, q4, first=first)
        assert q4.len == n and (q4.k_codes == 3).all()
        dar.dar_cache_unpack_q4(q4, src, first=first)
        assert src.len == n and (src.k_lat == 0).all()


def paged_pair(g, lens, ps, ps4, dd, dtype, w, d=64, Hkv=2, extra=0):
    """A cache of latent pages and one of 4-bit pages for sequences of `lens` tokens,
    with page sizes and tables of their own."""
    B = len(lens)
    most = max(max(lens), 1) + extra
    caches = []
    for cls, p in ((dar.DarPagedCache, ps), (dar.DarPagedCacheQ4, ps4)):
        maxb = -(-most // p)
        c = cls(B, Hkv, d, dd, w, p, maxb, B * maxb + 3, dtype)
        c.block_table.copy_(torch.randperm(B * maxb + 3, generator=g)[:B * maxb].reshape(B, maxb).to(torch.int32))
        c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        caches.append(c)
    return caches


def rows_of(c, pool, b, n):
    """Rows [Hkv, n, width] of sequence b's first n tokens."""
    e = torch.arange(n, device="cuda")
    return pool[c.block_table[b, e // c.page_size].long(), :, e % c.page_size].transpose(0, 1)


@pytest.mark.parametrize("dtype,dd,ps,ps4", [(BF, 16, 64, 32), (BF, 32, 32, 128), (F32, 16, 64, 64), (F32, 40, 32, 64)])
def test_pack_and_unpack_paged(dtype, dd, ps, ps4):
    g = gen(dd + ps)
    w, lens = 6, [300, 7, 0, -5, 6, 65, 1]
    src, q4 = paged_pair(g, lens, ps, ps4, dd, dtype, w)
    first = torch.tensor([40, 0, 0, 0, 0, 64, 9], dtype=torch.int32).cuda()
    src.k_pool.copy_(randn(g, *src.k_pool.shape, dtype=dtype))
    src.v_pool.copy_(randn(g, *src.v_pool.shape, dtype=dtype))
    q4.lens.fill_(77)
    for f in (None, first):
        for t in (q4.k_codes, q4.v_codes, q4.k_exp, q4.v_exp):
            t.fill_(0xA5)
        dar.dar_cache_pack_paged_q4(src, q4, first=f)
        assert q4.lens.cpu().tolist() == lens
        touched = torch.zeros(q4.n_pages, q4.page_size, dtype=torch.bool, device="cuda")
        for b, n in enumerate(lens):
            f0, D = (int(first[b]) if f is not None else 0), max(n - w, 0)
            if D <= f0:
                continue
            e = torch.arange(f0, D, device="cuda")
            touched[q4.block_table[b, e // ps4].long(), e % ps4] = True
            for pool, codes, exps in ((src.k_pool, q4.k_codes, q4.k_exp), (src.v_pool, q4.v_codes, q4.v_exp)):
                check_rows(rows_of(q4, codes, b, D)[:, f0:], rows_of(q4, exps, b, D)[:, f0:],
                           rows_of(src, pool, b, D)[:, f0:], dd)
        for t in (q4.k_codes, q4.v_codes, q4.k_exp, q4.v_exp):
            assert (t.transpose(1, 2)[~touched] == 0xA5).all()
        back = dar.DarPagedCache(len(lens), 2, 64, dd, w, ps, src.max_blocks, src.n_pages, dtype)
        back.block_table.copy_(src.block_table)
        dar.dar_cache_unpack_paged_q4(q4, back, first=f)
        assert back.lens.cpu().tolist() == lens
        for b, n in enumerate(lens):
            f0, D = (int(first[b]) if f is not None else 0), max(n - w, 0)
            if D > f0:
                got = f64(rows_of(back, back.k_pool, b, D)[:, f0:]).reshape(-1, dd)
                c = rows_of(q4, q4.k_codes, b, D)[:, f0:].cpu().numpy()
                e = rows_of(q4, q4.k_exp, b, D)[:, f0:].cpu().numpy()
                assert np.array_equal(got, ref.values(c.reshape(-1, c.shape[2]), e.reshape(-1, e.shape[2]), dd))


@pytest.mark.parametrize("dtype,dd", [(BF, 16), (F32, 20)])
def test_paged_conversion_limits(dtype, dd):
    """Unmapped pages on either side, a sequence that the destination does not hold,
    and lengths kept in one array."""
    g = gen(9)
    w, lens = 4, [200, 100, 90]
    src, q4 = paged_pair(g, lens, 32, 32, dd, dtype, w)
    src.k_pool.copy_(randn(g, *src.k_pool.shape, dtype=dtype))
    src.v_pool.copy_(randn(g, *src.v_pool.shape, dtype=dtype))
    src.block_table[0, 1] = -1
    src.block_table[1, 2] = src.n_pages
    q4.block_table[0, 3] = q4.n_pages + 9
    small = dar.DarPagedCacheQ4(3, 2, 64, dd, w, 32, 4, 12, dtype)       # 128 tokens a sequence
    small.block_table.copy_(torch.arange(12).reshape(3, 4).to(torch.int32))
    for t in (q4.k_codes, q4.k_exp, small.k_codes):
        t.fill_(0xA5)
    q4.share_ring(src)
    assert q4.lens is src.lens
    dar.dar_cache_pack_paged_q4(src, q4)
    assert src.lens.cpu().tolist() == lens
    e = rows_of(q4, q4.k_exp, 0, 96)
    assert (e[:, 32:64] == 3).all() and (e[:, :32] != 3).all()           # zeros from an unmapped page
    assert (rows_of(q4, q4.k_codes, 0, 64)[:, 32:] == 0).all()
    used = torch.zeros(q4.n_pages, dtype=torch.bool)
    bt = q4.block_table.cpu()
    for b, n in enumerate(lens):
        for k in range(-(-(n - w) // 32)):
            if 0 <= bt[b, k] < q4.n_pages:
                used[bt[b, k]] = True
    assert (q4.k_codes[~used.cuda()] == 0xA5).all()
    dar.dar_cache_pack_paged_q4(src, small)
    assert small.lens.cpu().tolist() == [-201, 100, 90] and small.overflowed() == [0]
    assert (small.k_codes[:4] == 0xA5).all() and (small.k_codes[4:7, :, :, :dd // 2] != 0xA5).any()


@pytest.mark.parametrize("dtype,dd", [(BF, 16), (BF, 32), (F32, 20)])
def test_paged_conversions_of_marked_lengths(dtype, dd):
    """Any negative length converts nothing: the lowest ones, too, from which w cannot be
    taken in 32 bits, and a first past every token."""
    g = gen(dd)
    least, w = -2 ** 31, 5
    lens = [70, least, least + 1, least + w, -1 - (1 << 30), -1, 40]
    src, q4 = paged_pair(g, lens, 32, 64, dd, dtype, w)
    back = dar.DarPagedCache(len(lens), 2, 64, dd, w, 32, src.max_blocks, src.n_pages, dtype)
    back.block_table.copy_(src.block_table)
    src.k_pool.copy_(randn(g, *src.k_pool.shape, dtype=dtype))
    src.v_pool.copy_(randn(g, *src.v_pool.shape, dtype=dtype))
    for first, held in (([0] * 7, {0: 65, 6: 35}), ([2 ** 31 - 1] * 6 + [0], {6: 35}), ([least] * 7, {0: 65, 6: 35})):
        first = torch.tensor(first, dtype=torch.int64).to(torch.int32).cuda()
        for t in (q4.k_codes, q4.v_codes, q4.k_exp, q4.v_exp):
            t.fill_(0xA5)
        for t in (back.k_pool, back.v_pool):
            t.fill_(17.0)
        q4.lens.zero_()
        dar.dar_cache_pack_paged_q4(src, q4, first=first)
        dar.dar_cache_unpack_paged_q4(q4, back, first=first)
        assert q4.lens.cpu().tolist() == back.lens.cpu().tolist() == lens
        for c, arrays, left in ((q4, (q4.k_codes, q4.v_codes, q4.k_exp, q4.v_exp), 0xA5), (back, (back.k_pool, back.v_pool), 17)):
            touched = torch.zeros(c.n_pages, c.page_size, dtype=torch.bool, device="cuda")
            for b, n in held.items():
                e = torch.arange(n, device="cuda")
                touched[c.block_table[b, e // c.page_size].long(), e % c.page_size] = True
            for t in arrays:
                assert (t.transpose(1, 2)[~touched] == left).all()
        for b, n in held.items():
            check_rows(rows_of(q4, q4.k_codes, b, n), rows_of(q4, q4.k_exp, b, n), rows_of(src, src.k_pool, b, n), dd)


@pytest.mark.parametrize("dtype,dd", [(BF, 16), (F32, 20)])
def test_paged_conversion_past_the_source(dtype, dd):
    """A length past what the source holds, which the destination would hold: nothing is
    converted, and the destination does not pass for one that has it."""
    g = gen(dd)
    w, lens = 4, [500, 96, 97, 50]
    for cls, other, arrays in ((dar.DarPagedCache, dar.DarPagedCacheQ4, ("k_codes", "v_codes", "k_exp", "v_exp")),
                               (dar.DarPagedCacheQ4, dar.DarPagedCache, ("k_pool", "v_pool"))):
        src = cls(4, 2, 64, dd, w, 32, 3, 12, dtype)                         # 96 tokens a sequence
        dst = other(4, 2, 64, dd, w, 64, 8, 32, dtype)                       # 512
        src.block_table.copy_(torch.randperm(12, generator=g).reshape(4, 3).to(torch.int32))
        dst.block_table.copy_(torch.randperm(32, generator=g).reshape(4, 8).to(torch.int32))
        src.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        for a in arrays:
            getattr(dst, a).fill_(7)
        (dar.dar_cache_pack_paged_q4 if cls is dar.DarPagedCache else dar.dar_cache_unpack_paged_q4)(src, dst)
        assert dst.lens.cpu().tolist() == [-501, 96, -98, 50]
        if other is dar.DarPagedCacheQ4:
            assert dst.overflowed() == [0, 2]
        for a in arrays:
            t = getattr(dst, a)
            for b, n in enumerate((0, 92, 0, 46)):
                assert (rows_of(dst, t, b, 512)[:, n:] == 7).all()
                assert n == 0 or (rows_of(dst, t, b, n) != 7).any()


# --- appends --------------------------------------------------------------------

SHAPES = [(64, 16, BF), (128, 32, BF), (64, 32, BF), (128, 16, BF), (64, 16, F32), (80, 20, F32), (48, 40, BF), (256, 96, F32),
          (33, 5, BF)]


@pytest.mark.parametrize("d,dd,dtype", SHAPES)
@pytest.mark.parametrize("w,pieces", [(16, [1, 5, 11, 1, 40, 16, 15, 17, 1]), (0, [3, 1, 70]), (1, [1, 1, 4, 1]),
                                      (100, [30, 60, 9, 1, 1, 250])])
def test_append_is_the_packed_append(d, dd, dtype, w, pieces):
    """Codes, scales and ring are those of dar_cache_append's latents, packed: however
    the tokens are batched."""
    B, Hkv = 2, 3
    g = gen(d + dd + w)
    n = sum(pieces)
    k, v = (randn(g, B, Hkv, n, d, dtype=dtype) for _ in range(2))
    wd = randn(g, Hkv, d, dd, dtype=dtype, std=d ** -0.5)
    plain = dar.DarCache(B, Hkv, d, dd, w, n, dtype)
    want = dar.DarCacheQ4(B, Hkv, d, dd, w, n, dtype)
    got = dar.DarCacheQ4(B, Hkv, d, dd, w, n, dtype)
    for t in (got.k_codes, got.v_codes, got.k_exp, got.v_exp, want.k_codes, want.v_codes, want.k_exp, want.v_exp):
        t.fill_(0xA5)
    at = 0
    for m in pieces:
        kk, vv = (x[:, :, at:at + m].contiguous() for x in (k, v))
        dar.dar_cache_append(plain, kk, vv, wd)
        dar.dar_cache_append_q4(got, kk, vv, wd)
        at += m
        assert got.len == at
        dar.dar_cache_pack_q4(plain, want)
        for a in ("k_codes", "v_codes", "k_exp", "v_exp"):
            assert torch.equal(getattr(got, a), getattr(want, a)), (a, at)
        if w:
            assert torch.equal(got.k_win, plain.k_win) and torch.equal(got.v_win, plain.v_win), at


@pytest.mark.parametrize("d,dd,dtype", SHAPES)
@pytest.mark.parametrize("w", [0, 1, 20])
def test_append_paged(d, dd, dtype, w):
    """Steps of a ragged batch against the dense append of every sequence; sequences
    at capacity, overflowed, and with an unmapped page are left as they are."""
    g = gen(d + w)
    lens, Hkv, ps, steps = [0, 5, w, 19, 63, 64, 70, 96, -4, 31], 3, 32, 3
    B = len(lens)
    c = dar.DarPagedCacheQ4(B, Hkv, d, dd, w, ps, 3, 3 * B + 1, dtype)   # 96 tokens a sequence
    c.block_table.copy_(torch.randperm(3 * B, generator=g).reshape(B, 3).to(torch.int32))
    c.block_table[6] = -1
    wd = randn(g, Hkv, d, dd, dtype=dtype, std=d ** -0.5)
    before = [randn(g, 1, Hkv, max(n, 1), d, dtype=dtype) for n in lens for _ in range(2)]
    new = [randn(g, steps, B, Hkv, d, dtype=dtype) for _ in range(2)]
    dense = []
    for t in (c.k_codes, c.v_codes, c.k_exp, c.v_exp):
        t.fill_(0xA5)
    for b, n in enumerate(lens):
        one = dar.DarCacheQ4(1, Hkv, d, dd, w, 128, dtype)
        if n > 0:
            dar.dar_cache_append_q4(one, before[2 * b], before[2 * b + 1], wd)
            if w:
                c.k_win[b], c.v_win[b] = one.k_win[0], one.v_win[0]
        dense.append(one)
    c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    start = [x.clone() for x in (c.k_codes, c.k_exp)]
    for t in range(steps):
        dar.dar_cache_append_paged_q4(c, new[0][t].clone(), new[1][t].clone(), wd)  # (aligned)
    now = [n + steps if 0 <= n <= 96 - steps else n for n in lens]
    now[7] = -97
    assert c.lens.cpu().tolist() == now
    touched = torch.zeros(c.n_pages, ps, dtype=torch.bool, device="cuda")
    for b, n in enumerate(lens):
        if n < 0 or n == 96:
            continue
        for t in range(steps):
            dar.dar_cache_append_q4(dense[b], new[0][t, b:b + 1, :, None].clone(),
                                    new[1][t, b:b + 1, :, None].clone(), wd)
        if w:
            assert torch.equal(c.k_win[b], dense[b].k_win[0]) and torch.equal(c.v_win[b], dense[b].v_win[0]), b
        D0, D = max(n - w, 0), max(n + steps - w, 0)
        if D == D0 or b == 6:
            continue
        e = torch.arange(D0, D, device="cuda")
        touched[c.block_table[b, e // ps].long(), e % ps] = True
        for a in ("k_codes", "v_codes", "k_exp", "v_exp"):
            assert torch.equal(rows_of(c, getattr(c, a), b, D)[:, D0:], getattr(dense[b], a)[0, :, D0:D]), (a, b)
    for x, s in zip((c.k_codes, c.k_exp), start):
        assert torch.equal(x.transpose(1, 2)[~touched], s.transpose(1, 2)[~touched])


# --- decode ----------------------------------------------------------------------

def filled(B, Hq, Hkv, d, dd, w, n, dtype, seed, untied=False, cap=None):
    """A dense 4-bit cache of n tokens, queries and weights; scales over a few powers
    of two, a few tokens attended far above the rest."""
    g = gen(seed)
    c = dar.DarCacheQ4(B, Hkv, d, dd, w, cap or n, dtype)
    lat = dar.DarCache(B, Hkv, d, dd, w, c.cap, dtype)
    for x in (lat.k_lat, lat.v_lat):
        x.copy_(randn(g, *x.shape, dtype=dtype) * torch.exp2(torch.randint(-2, 2, (*x.shape[:3], 1), generator=g).float()).cuda())
    lat.struct.len = n
    for t in (c.k_codes, c.v_codes, c.k_exp, c.v_exp):
        t.fill_(0xFF)                           # what lies past the end must not be met
    dar.dar_cache_pack_q4(lat, c)
    c.k_win.copy_(randn(g, *c.k_win.shape, dtype=dtype))
    c.v_win.copy_(randn(g, *c.v_win.shape, dtype=dtype))
    q = randn(g, B, Hq, d, dtype=dtype, std=2.0)
    wd = randn(g, Hkv, d, dd, dtype=dtype, std=d ** -0.5)
    wu = randn(g, Hkv, dd, d, dtype=dtype, std=dd ** -0.5) if untied else None
    return c, q, wd, wu


def check_step(o, q, codes, rings, wd, wu, lens, w, dtype):
    """o [B,Hq,d] against the reference; codes(b, g, n): key and value rows."""
    B, Hq, d = o.shape
    Hkv, dd = wd.shape[0], wd.shape[2]
    G = Hq // Hkv
    up = f64(wd).transpose(0, 2, 1) if wu is None else f64(wu)
    for b, n in enumerate(lens):
        for g in range(Hkv):
            hs = slice(g * G, (g + 1) * G)
            k, v = codes(b, g, max(n - w, 0))
            want, mass, terms = ref.decode(f64(q)[b, hs], k, v, f64(rings[0][b, g]), f64(rings[1][b, g]), up[g], n, w)
            off = np.abs(f64(o[b, hs]) - want)
            most = ref.decode_atol(want, mass, terms, n, d, dd, dtype == BF)
            assert (off <= most).all(), (b, g, float((off / most).max()))


def dense_codes(c):
    def get(b, g, n):
        dd = c.d_down
        return tuple(ref.values(x[b, g, :n].cpu().numpy(), e[b, g, :n].cpu().numpy(), dd)
                     for x, e in ((c.k_codes, c.k_exp), (c.v_codes, c.v_exp)))
    return get


@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (4, 2), (3, 1), (8, 2), (5, 1), (14, 2), (8, 1), (12, 1), (17, 1)])
@pytest.mark.parametrize("d,dd,untied", [(64, 16, False), (128, 32, True), (64, 32, True), (128, 16, False)])
def test_decode_heads(Hq, Hkv, d, dd, untied):
    n, w = 700, 37
    c, q, wd, wu = filled(2, Hq, Hkv, d, dd, w, n, BF, Hq + d, untied)
    o = dar.dar_attn_decode_q4(c, q, wd, wu) if wu is not None else dar.dar_attn_decode_q4(c, q, wd)
    check_step(o, q, dense_codes(c), (c.k_win, c.v_win), wd, wu, [n] * 2, w, BF)


@pytest.mark.parametrize("d,dd,dtype,Hq", [(64, 16, BF, 8), (128, 32, BF, 16), (80, 20, F32, 8), (64, 16, F32, 2),
                                           (48, 40, BF, 6), (256, 128, F32, 4), (33, 5, BF, 2)])
@pytest.mark.parametrize("w,n", [(32, 1), (32, 2), (32, 31), (32, 32), (32, 33), (32, 34), (32, 160), (32, 161), (0, 1),
                                 (0, 127), (0, 300), (1, 1), (1, 2), (7, 4000), (300, 290), (300, 1111), (513, 70000)])
def test_decode_lengths(d, dd, dtype, Hq, w, n):
    if n > 5000 and dtype == F32 and d == 256:
        n = 5001
    c, q, wd, wu = filled(1, Hq, 2, d, dd, w, n, dtype, n + w + d, cap=n + 130)
    o = dar.dar_attn_decode_q4(c, q, wd)
    check_step(o, q, dense_codes(c), (c.k_win, c.v_win), wd, wu, [n], w, dtype)


@pytest.mark.parametrize("d,dd,dtype", [(64, 16, BF), (128, 32, BF), (64, 32, BF), (80, 20, F32)])
@pytest.mark.parametrize("ps,extra", [(32, 0), (64, 0), (256, 0), (32, 9000), (64, 9000), (128, 9000)])
def test_decode_paged(d, dd, dtype, ps, extra):
    """extra: room past the longest sequence; with it no pair is one workgroup's."""
    g = gen(ps + d)
    w, Hq, Hkv = 45, 8, 2
    lens = [900, 1, 0, 45, 46, 333, 1500, -7, 64, 205]
    _, c = paged_pair(g, lens, 32, ps, dd, dtype, w, d=d, extra=extra)
    B = len(lens)
    for k, e in ((c.k_codes, c.k_exp), (c.v_codes, c.v_exp)):
        k.copy_(torch.randint(0, 256, k.shape, generator=g, dtype=torch.uint8))
        e.copy_(torch.randint(125, 129, e.shape, generator=g, dtype=torch.uint8))
    # pages that no sequence holds, and rows past the ends
    live = torch.zeros(c.n_pages, ps, dtype=torch.bool, device="cuda")
    for b, n in enumerate(lens):
        at = torch.arange(max(n - w, 0), device="cuda")
        live[c.block_table[b, at // ps].long(), at % ps] = True
    for e in (c.k_exp, c.v_exp):
        e.transpose(1, 2)[~live] = 255
    c.block_table[5, 1] = -1                  # reads as zeros
    c.block_table[6, 0] = c.n_pages
    c.k_win.copy_(randn(g, *c.k_win.shape, dtype=dtype))
    c.v_win.copy_(randn(g, *c.v_win.shape, dtype=dtype))
    q = randn(g, B, Hq, d, dtype=dtype, std=2.0)
    wd = randn(g, Hkv, d, dd, dtype=dtype, std=d ** -0.5)
    wu = randn(g, Hkv, dd, d, dtype=dtype, std=dd ** -0.5)
    o = dar.dar_attn_decode_paged_q4(c, q, wd, wu)
    bt = c.block_table.cpu().numpy()

    def codes(b, gk, n):
        out = []
        for x, e in ((c.k_codes, c.k_exp), (c.v_codes, c.v_exp)):
            pages = bt[b, np.arange(n) // ps]
            ok = (pages >= 0) & (pages < c.n_pages)
            at = np.where(ok, pages, 0), gk, np.arange(n) % ps
            v = ref.values(x.cpu().numpy()[at], e.cpu().numpy()[at], dd)
            out.append(np.where(ok[:, None], v, 0.0))
        return out
    some = [b for b, n in enumerate(lens) if n > 0]
    check_step(o[some], q[some], lambda i, gk, n: codes(some[i], gk, n), (c.k_win[some], c.v_win[some]), wd, wu,
               [lens[b] for b in some], w, dtype)
    assert torch.isnan(o[2]).all() and torch.isnan(o[7]).all()


@pytest.mark.parametrize("d,dd,dtype,blocks", [(64, 16, BF, 3), (64, 16, BF, 600), (128, 32, BF, 600),
                                               (80, 20, F32, 3), (80, 20, F32, 600)])
def test_decode_many_sequences(d, dd, dtype, blocks):
    """More sequences than a wavefront has lanes, more pairs than wavefronts, lengths
    from none to past what is mapped; blocks: of a sequence's table, three mapped."""
    B, Hq, Hkv, w, ps = 1100, 4, 4, 8, 32
    g = gen(B)
    lens = torch.randint(0, 97, (B,), generator=g)
    lens[::97] = 0
    lens[5], lens[6] = -3, 500 if blocks == 3 else 90     # (past its capacity: read up to it)
    c = dar.DarPagedCacheQ4(B, Hkv, d, dd, w, ps, blocks, 3 * B, dtype)
    c.block_table[:, :3].copy_(torch.arange(3 * B).reshape(B, 3).to(torch.int32))
    c.lens.copy_(lens.to(torch.int32))
    for k, e in ((c.k_codes, c.k_exp), (c.v_codes, c.v_exp)):
        k.copy_(torch.randint(0, 256, k.shape, generator=g, dtype=torch.uint8))
        e.copy_(torch.randint(125, 129, e.shape, generator=g, dtype=torch.uint8))
    c.k_win.copy_(randn(g, *c.k_win.shape, dtype=dtype))
    c.v_win.copy_(randn(g, *c.v_win.shape, dtype=dtype))
    q = randn(g, B, Hq, d, dtype=dtype, std=2.0)
    wd = randn(g, Hkv, d, dd, dtype=dtype, std=d ** -0.5)
    o = dar.dar_attn_decode_paged_q4(c, q, wd)
    held = lens.clamp(max=96).tolist()
    none = [b for b in range(B) if held[b] < 1]
    assert torch.isnan(o[none]).all() and torch.isfinite(o).all(2).all(1).sum() == B - len(none)
    some = [b for b in range(0, B, 7) if held[b] > 0] + [6]

    def codes(i, gk, n):
        b = some[i]
        return [ref.values(x[3 * b:3 * b + 3, gk].reshape(96, -1)[:n].cpu().numpy(),
                           e[3 * b:3 * b + 3, gk].reshape(96, -1)[:n].cpu().numpy(), dd)
                for x, e in ((c.k_codes, c.k_exp), (c.v_codes, c.v_exp))]
    check_step(o[some], q[some], codes, (c.k_win[some], c.v_win[some]), wd, None, [held[b] for b in some], w, dtype)


def paged_step(g, lens, Hq, Hkv, d, dd, dtype, w, ps, extra, untied):
    """A paged 4-bit cache of random codes, with scales that read as NaN wherever no
    sequence's distant token lies; a step over it, and codes(b, g, n) for check_step."""
    _, c = paged_pair(g, lens, 32, ps, dd, dtype, w, d=d, Hkv=Hkv, extra=extra)
    for k, e in ((c.k_codes, c.k_exp), (c.v_codes, c.v_exp)):
        k.copy_(torch.randint(0, 256, k.shape, generator=g, dtype=torch.uint8))
        e.copy_(torch.randint(125, 129, e.shape, generator=g, dtype=torch.uint8))
    live = torch.zeros(c.n_pages, ps, dtype=torch.bool, device="cuda")
    for b, n in enumerate(lens):
        at = torch.arange(max(n - w, 0), device="cuda")
        live[c.block_table[b, at // ps].long(), at % ps] = True
    for e in (c.k_exp, c.v_exp):
        e.transpose(1, 2)[~live] = 255
    c.k_win.copy_(randn(g, *c.k_win.shape, dtype=dtype))
    c.v_win.copy_(randn(g, *c.v_win.shape, dtype=dtype))
    q = randn(g, len(lens), Hq, d, dtype=dtype, std=2.0)
    wd = randn(g, Hkv, d, dd, dtype=dtype, std=d ** -0.5)
    wu = randn(g, Hkv, dd, d, dtype=dtype, std=dd ** -0.5) if untied else None

    def codes(b, gk, n):
        return [ref.values(rows_of(c, x, b, n)[gk].cpu().numpy(), rows_of(c, e, b, n)[gk].cpu().numpy(), dd)
                for x, e in ((c.k_codes, c.k_exp), (c.v_codes, c.v_exp))]
    return c, q, wd, wu, codes


MANY_HEADS = [(5, 1), (14, 2), (8, 1), (12, 1), (17, 1), (50, 2)]


@pytest.mark.parametrize("Hq,Hkv", MANY_HEADS)
@pytest.mark.parametrize("d,dd,dtype,untied", [(64, 16, BF, False), (128, 32, BF, True), (64, 32, BF, True),
                                               (128, 16, BF, False), (80, 20, F32, False), (48, 40, BF, True)])
def test_decode_heads_by_records(Hq, Hkv, d, dd, dtype, untied):
    """More query heads a KV head than a tile has, with records and a merge (lengths
    past what one workgroup takes), and outside the matrix-core shapes."""
    n, w = 6000, 37
    c, q, wd, wu = filled(2, Hq, Hkv, d, dd, w, n, dtype, Hq + d, untied)
    o = dar.dar_attn_decode_q4(c, q, wd, wu)
    check_step(o, q, dense_codes(c), (c.k_win, c.v_win), wd, wu, [n] * 2, w, dtype)


@pytest.mark.parametrize("Hq,Hkv", [(4, 4)] + MANY_HEADS)
@pytest.mark.parametrize("d,dd,dtype", [(64, 16, BF), (128, 32, BF), (64, 32, BF), (128, 16, BF), (80, 20, F32), (33, 5, BF)])
@pytest.mark.parametrize("extra", [0, 9000])
def test_decode_paged_heads(Hq, Hkv, d, dd, dtype, extra):
    """Every paged form, by one launch (bf16 matrix shapes without extra) and by records."""
    lens = [700, 1, 37, 38, 300, 1500]
    c, q, wd, wu, codes = paged_step(gen(Hq + d), lens, Hq, Hkv, d, dd, dtype, 37, 64, extra, d == 64)
    o = dar.dar_attn_decode_paged_q4(c, q, wd, wu)
    check_step(o, q, codes, (c.k_win, c.v_win), wd, wu, lens, 37, dtype)


@pytest.mark.parametrize("d,dd,dtype", [(256, 160, F32), (256, 256, F32), (200, 129, BF), (256, 193, BF)])
@pytest.mark.parametrize("n,w", [(1, 0), (40, 33), (170, 33), (5000, 33), (9000, 0)])
def test_decode_wide_latents(d, dd, dtype, n, w):
    """Bottlenecks of five to eight groups of columns, dense (few heads with many
    records) and paged (many heads)."""
    c, q, wd, wu = filled(1, 6, 1, d, dd, w, n, dtype, d + dd, n % 2 == 0)
    o = dar.dar_attn_decode_q4(c, q, wd, wu)
    check_step(o, q, dense_codes(c), (c.k_win, c.v_win), wd, wu, [n], w, dtype)
    if n < 1000:
        lens = [n, 1, n + 64, 150] * 8
        c, q, wd, wu, codes = paged_step(gen(n), lens, 10, 5, d, dd, dtype, w, 32, 0, n % 2 == 0)
        o = dar.dar_attn_decode_paged_q4(c, q, wd, wu)
        check_step(o, q, codes, (c.k_win, c.v_win), wd, wu, lens, w, dtype)


@pytest.mark.parametrize("d,dd,dtype", [(64, 16, BF), (128, 32, BF), (80, 20, F32)])
@pytest.mark.parametrize("extra", [0, 100000])
def test_decode_one_long_among_short(d, dd, dtype, extra):
    """A table far longer than its sequences, or as long as the one long sequence."""
    lens = [40, 33, 90, 8000] + [50 + b for b in range(8)]
    c, q, wd, wu, codes = paged_step(gen(d), lens, 4, 2, d, dd, dtype, 32, 128, extra, False)
    o = dar.dar_attn_decode_paged_q4(c, q, wd)
    check_step(o, q, codes, (c.k_win, c.v_win), wd, None, lens, 32, dtype)


@pytest.mark.parametrize("dtype,dd,n,B,Hq,Hkv", [(BF, 16, 50, 1030, 64, 4), (BF, 16, 17000, 4, 16500, 1),
                                                  (F32, 12, 50, 1030, 64, 4)])
def test_many_query_heads(dtype, dd, n, B, Hq, Hkv):
    """More than 65535 query heads in a batch of fewer KV heads: a step, as one launch
    (bf16, 50 tokens) and with records, and an append."""
    d, w, G = 64, 16, Hq // Hkv
    assert B * Hq > 65535
    c, q, wd, _ = filled(B, Hq, Hkv, d, dd, w, n, dtype, 11, cap=n + 1)
    o = dar.dar_attn_decode_q4(c, q, wd)
    assert torch.isfinite(o).all()
    some = [0, 1, B - 1]
    heads = [g * G + h for g in range(Hkv) for h in (0, 7, 8, G // 2, G - 1)]
    get = dense_codes(c)
    check_step(o[some][:, heads], q[some][:, heads], lambda i, g, m: get(some[i], g, m), (c.k_win[some], c.v_win[some]),
               wd, None, [n] * 3, w, dtype)
    # the append, at the shape with all query heads, against the 16-bit one packed
    plain = dar.DarCache(B, Hkv, d, dd, w, c.cap, dtype)
    plain.k_win.copy_(c.k_win)
    plain.v_win.copy_(c.v_win)
    plain.struct.len = n
    g = gen(12)
    k, v = (randn(g, B, Hkv, 1, d, dtype=dtype) for _ in range(2))
    shape = dar.make_shape(B, Hq, Hkv, d, dd, w, dtype)
    assert dar.lib.dar_cache_append_q4(shape, c.struct, k.data_ptr(), v.data_ptr(), 1, wd.data_ptr(), None) == dar.DAR_OK
    dar.dar_cache_append(plain, k, v, wd)
    want = dar.DarCacheQ4(B, Hkv, d, dd, w, c.cap, dtype)
    dar.dar_cache_pack_q4(plain, want, first=n - w)
    assert c.len == n + 1 and torch.equal(c.k_win, plain.k_win) and torch.equal(c.v_win, plain.v_win)
    for a in ("k_codes", "v_codes", "k_exp", "v_exp"):
        assert torch.equal(getattr(c, a)[:, :, n - w], getattr(want, a)[:, :, n - w])


@pytest.mark.parametrize("d,dd,dtype", [(64, 16, BF), (128, 32, BF), (80, 20, F32)])
@pytest.mark.parametrize("which", ["k_exp", "v_exp"])
def test_nan_latents_stay_with_their_head(d, dd, dtype, which):
    """A latent that reads as NaN makes its KV head's outputs NaN, in its sequence only."""
    c, q, wd, _ = filled(2, 8, 2, d, dd, 16, 500, dtype, 3)
    want = dar.dar_attn_decode_q4(c, q, wd)
    getattr(c, which)[1, 0, 333] = 255
    getattr(c, which.replace("exp", "codes"))[1, 0, 333] = 0
    o = dar.dar_attn_decode_q4(c, q, wd)
    assert torch.isnan(o[1, :4]).all()
    assert torch.equal(o[0], want[0]) and torch.equal(o[1, 4:], want[1, 4:])


@pytest.mark.parametrize("d,dd,dtype", [(64, 16, BF), (128, 32, BF), (80, 20, F32)])
@pytest.mark.parametrize("w,n,at", [(0, 1, 0), (16, 129 + 16, 128), (16, 6401 + 16, 6400), (16, 20, 3)])
def test_nan_latent_alone(d, dd, dtype, w, n, at):
    """The same where the token is the only one of its block, or of the cache."""
    c, q, wd, _ = filled(2, 4, 1, d, dd, w, n, dtype, 3)
    c.k_exp[1, 0, at] = 255
    c.k_codes[1, 0, at] = 0
    o = dar.dar_attn_decode_q4(c, q, wd)
    assert torch.isnan(o[1]).all() and torch.isfinite(o[0]).all()
    q[0, 2, 5] = float("nan")                  # and a query's
    o = dar.dar_attn_decode_q4(c, q, wd)
    assert torch.isnan(o[0, 2]).all() and torch.isfinite(o[0, [0, 1, 3]]).all()


@pytest.mark.parametrize("d,dd,dtype", [(64, 16, BF), (80, 20, F32)])
def test_large_scores_and_scales(d, dd, dtype):
    """Scores in the hundreds that rise along the cache (the reference moves again
    and again), and values at scales 2^-60 and 2^60."""
    n, w = 2000, 16
    c, q, wd, _ = filled(1, 4, 1, d, dd, w, n, dtype, 5)
    c.k_exp[0, 0, :n - w] = (120 + torch.arange(n - w) * 14 // n).to(torch.uint8).cuda()[:, None]
    c.v_exp[0, 0, :n - w] = (67 + 120 * (torch.arange(n - w) % 2)).to(torch.uint8).cuda()[:, None]
    o = dar.dar_attn_decode_q4(c, q, wd)
    check_step(o, q, dense_codes(c), (c.k_win, c.v_win), wd, None, [n], w, dtype)


def test_long_cache():
    """2^27 tokens in each of 3 KV heads: byte offsets far past 2^32 (two arrays of
    6 GiB). One token near the end takes all the weight."""
    d, dd, w, n = 128, 32, 64, (1 << 27) - 63
    c = dar.DarCacheQ4(1, 3, d, dd, w, n, BF)
    c.k_exp.fill_(127)
    c.v_exp.fill_(127)
    g = gen(1)
    q = randn(g, 1, 3, d)
    wd = randn(g, 3, d, dd, std=d ** -0.5)
    qt = torch.bmm(q[0, :, None].float(), wd.float())[:, 0]
    at = [n - w - 1, n - w - 130, 3]
    for h, e in enumerate(at):
        nib = torch.where(qt[h] < 0, 15, 7).to(torch.uint8)              # +-6 by the query's sign
        c.k_codes[0, h, e] = nib[0::2] | (nib[1::2] << 4)
        c.k_exp[0, h, e] = 127 + 8
        c.v_codes[0, h, e] = 0x22                                          # ones
    c.struct.len = n
    c.k_win.copy_(randn(g, *c.k_win.shape))
    c.v_win.copy_(randn(g, *c.v_win.shape))
    o = dar.dar_attn_decode_q4(c, q, wd)
    want = wd.double().sum(2)
    assert (o[0].double() - want).abs().max() <= (2.0 ** -8 + 2.0 ** -14) * want.abs().max()
    k = randn(g, 1, 3, 2, d)
    before = c.k_win.clone()
    c.struct.len = n - 2                      # two tokens leave, at slots near 2^27
    dar.dar_cache_append_q4(c, k, k, wd)
    slots = torch.arange(n - 2 - w, n - w, device="cuda") % w
    x = torch.bmm(before[0][:, slots].float(), wd.float()).to(BF)
    codes, exps = ref.quantise(f64(x).reshape(-1, dd))
    got = c.k_exp[0, :, n - 2 - w:n - w].cpu().numpy().reshape(-1, 1)
    assert (np.abs(got.astype(int) - exps) <= 1).all()                      # (fp32 sums in another order)


@pytest.mark.parametrize("d,dd,dtype", [(128, 32, BF), (64, 33, F32)])
def test_long_cache_writes(d, dd, dtype):
    """Rows past 2^28, whose codes lie past byte 2^32: an append, its read-back and the
    pack of that, each against a short cache with the same slots, to the byte, and
    nothing else written."""
    w, n = 64, (1 << 28) + 61                 # two tokens leave: slots n - w, n - w + 1
    short = 128 + n % w                       # the same place in the ring
    g = gen(dd)
    wd = randn(g, 1, d, dd, dtype=dtype, std=d ** -0.5)
    new = [randn(g, 1, 1, 2, d, dtype=dtype) for _ in range(2)]
    ring = [randn(g, 1, 1, w, d, dtype=dtype) for _ in range(2)]
    held = []
    names = ("k_codes", "v_codes", "k_exp", "v_exp")
    for m in (short, n):
        c = dar.DarCacheQ4(1, 1, d, dd, w, m + 2, dtype)
        for a in names:
            getattr(c, a).fill_(0xA5)
        c.k_win.copy_(ring[0])
        c.v_win.copy_(ring[1])
        c.struct.len = m
        dar.dar_cache_append_q4(c, new[0], new[1], wd)
        back = dar.DarCache(1, 1, d, dd, w, m + 2, dtype)
        dar.dar_cache_unpack_q4(c, back, first=m - w)
        again = dar.DarCacheQ4(1, 1, d, dd, w, m + 2, dtype)
        dar.dar_cache_pack_q4(back, again, first=m - w)
        at = slice(m - w, m - w + 2)
        for x in (c.k_codes, c.v_codes):
            assert (x[0, 0, at, :dd // 2] != 0xA5).any()
        for x, left in [(getattr(c, a), 0xA5) for a in names] + [(getattr(again, a), 0) for a in names] + [
                (back.k_lat, 0), (back.v_lat, 0)]:
            for lo in range(0, x.shape[2], 1 << 24):   # (in pieces: comparisons take as much memory again)
                piece = x[0, 0, lo:lo + (1 << 24)] != left
                keep = torch.ones(len(piece), dtype=torch.bool, device="cuda")
                keep[max(at.start - lo, 0):max(at.stop - lo, 0)] = False
                assert not piece.any(1).logical_and_(keep).any(), (m, lo)
        held.append([getattr(x, a)[0, 0, at].clone() for x in (c, again) for a in names] +
                    [back.k_lat[0, 0, at].clone(), back.v_lat[0, 0, at].clone(), c.k_win.clone(), c.v_win.clone()])
        del c, back, again, x, piece
    for i, (x, y) in enumerate(zip(*held)):
        assert torch.equal(x, y), i


# --- together ----------------------------------------------------------------------

@pytest.mark.parametrize("d,dd,w,dtype", [(64, 16, 32, BF), (128, 32, 48, BF), (80, 20, 16, F32)])
def test_turns_of_a_conversation(d, dd, w, dtype):
    """A prompt prefilled into a cache and packed, decode steps on the 4-bit cache,
    read back for the next prompt's chunk, packed on, and more steps: every
    step's output against the cache's own contents, which follow the tokens."""
    B, Hq, Hkv, n0, n1, steps = 2, 8, 2, 150, 70, 20
    g = gen(d)
    wd = randn(g, Hkv, d, dd, dtype=dtype, std=d ** -0.5)
    cap = n0 + n1 + 2 * steps
    plain = dar.DarCache(B, Hkv, d, dd, w, cap, dtype)
    q4 = dar.DarCacheQ4(B, Hkv, d, dd, w, cap, dtype).share_ring(plain)
    ks, vs, first = [], [], 0

    def tokens(n):
        k, v = (randn(g, B, Hkv, n, d, dtype=dtype) for _ in range(2))
        ks.append(k)
        vs.append(v)
        return k, v

    for turn, n in enumerate((n0, n1)):
        k, v = tokens(n)
        dar.dar_attn_prefill_chunk(plain, randn(g, B, Hq, n, d, dtype=dtype), k, v, wd)
        dar.dar_cache_pack_q4(plain, q4, first=first)
        for _ in range(steps):
            k, v = tokens(1)
            dar.dar_cache_append_q4(q4, k, v, wd)
            q = randn(g, B, Hq, d, dtype=dtype, std=2.0)
            o = dar.dar_attn_decode_q4(q4, q, wd)
            check_step(o, q, dense_codes(q4), (q4.k_win, q4.v_win), wd, None, [q4.len] * B, w, dtype)
        n = q4.len
        kk, vv = torch.cat(ks, 2), torch.cat(vs, 2)
        slots = torch.arange(n - w, n, device="cuda") % w
        assert torch.equal(q4.k_win[:, :, slots], kk[:, :, n - w:]) and torch.equal(q4.v_win[:, :, slots], vv[:, :, n - w:])
        # the codes are those of the tokens: within half a step of the format and the
        # rounding of the latent (2^-8 of it), or 1/7 where a value saturates
        lat = torch.matmul(kk[:, :, :n - w].double(), wd.double()).cpu().numpy()
        for b in range(B):
            for h in range(Hkv):
                got = dense_codes(q4)(b, h, n - w)[0]
                s = 2.0 ** (q4.k_exp[b, h, :n - w, 0].cpu().numpy().astype(float) - 127)
                assert (np.abs(got - lat[b, h]) <= s[:, None] * 1.0 + 2.0 ** -7 * np.abs(lat[b, h])).all()
        dar.dar_cache_unpack_q4(q4, plain, first=first)
        assert plain.len == n
        first = n - w


def batch(seed=4, lens=(900, 5, 0, 300, 64, 1200)):
    g = gen(seed)
    B, Hq, Hkv, d, dd, w, ps = len(lens), 8, 2, 64, 16, 32, 64
    maxb = max(lens) // ps + 2
    c = dar.DarPagedCacheQ4(B, Hkv, d, dd, w, ps, maxb, B * maxb, BF)
    c.block_table.copy_(torch.randperm(B * maxb, generator=g).reshape(B, maxb).to(torch.int32))
    for t in (c.k_codes, c.v_codes):
        t.copy_(torch.randint(0, 256, t.shape, generator=g, dtype=torch.uint8))
    c.k_exp.fill_(126)
    c.v_exp.fill_(126)
    for t in (c.k_win, c.v_win):
        t.copy_(torch.randn(t.shape, generator=g))
    c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    back = dar.DarPagedCache(B, Hkv, d, dd, w, ps, maxb, B * maxb, BF)
    back.block_table.copy_(c.block_table)
    return (c, back, randn(g, B, Hq, d, std=2.0), randn(g, Hkv, d, dd, std=0.125),
            [randn(g, B, Hkv, d) for _ in range(2)])


def held(u, *more):
    c, back = u[:2]
    return [x.clone() for x in (c.k_win, c.v_win, c.k_codes, c.v_codes, c.k_exp, c.v_exp, c.lens, back.k_pool,
                                back.v_pool, back.lens, *more)]


def restore(u, saved):
    c, back = u[:2]
    for t, x in zip((c.k_win, c.v_win, c.k_codes, c.v_codes, c.k_exp, c.v_exp, c.lens, back.k_pool, back.v_pool,
                     back.lens), saved):
        t.copy_(x)


def same(a, b):
    return all(torch.equal(x.view(torch.int16) if x.dtype == BF else x, y.view(torch.int16) if y.dtype == BF else y)
               for x, y in zip(a, b))


def step(u, o=None, ws=None, stream=None):
    c, back, q, wd, new = u
    dar.dar_cache_append_paged_q4(c, new[0], new[1], wd, stream=stream)
    o = dar.dar_attn_decode_paged_q4(c, q, wd, o=o, ws=ws, stream=stream)
    dar.dar_cache_unpack_paged_q4(c, back, stream=stream)
    dar.dar_cache_pack_paged_q4(back, c, stream=stream)
    return o


def workspace(*users):
    return torch.empty(max(dar.dar_decode_q4_workspace_bytes(
        dar.make_shape(u[0].B, u[2].shape[1], u[0].Hkv, u[0].d, u[0].d_down, u[0].w, BF), u[0].cap) for u in users),
        dtype=torch.uint8, device="cuda")


def test_graphs_share_a_workspace():
    """Two captured steps of different batches over one workspace, replayed with eager
    steps between: each ends where its eager step ended."""
    users = [batch(), batch(seed=6, lens=(700, 1100, 301, 0, 1, 288))]
    ws = workspace(*users)
    starts, ends, outs, graphs = [], [], [torch.empty_like(u[2]) for u in users], []
    for u, o in zip(users, outs):
        starts.append(held(u))
        step(u, o, ws)
        torch.cuda.synchronize()
        ends.append(held(u, o))
        restore(u, starts[-1])
        graph, cs = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        cs.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(cs):
            with torch.cuda.graph(graph, stream=cs):
                step(u, o, ws)
        torch.cuda.current_stream().wait_stream(cs)
        graphs.append(graph)
    other = batch(seed=8)
    for rep in range(3):
        for u, s0, o in zip(users, starts, outs):
            restore(u, s0)
            o.fill_(float("nan"))
        step(other, ws=ws)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for u, o, end in zip(users, outs, ends):
            assert same(held(u, o), end), rep


def test_other_streams():
    """Two batches on two streams at once, with outputs and workspaces of the calls'
    own, while the default stream goes on allocating and writing."""
    users = [batch(seed=6), batch(seed=7)]
    ends = []
    for u in users:
        s0 = held(u)
        o = step(u)
        torch.cuda.synchronize()
        ends.append(held(u, o))
        restore(u, s0)
    need = workspace(*users).numel()
    streams = [torch.cuda.Stream() for _ in users]
    torch.cuda.synchronize()
    got, busy = [], []
    for u, s in zip(users, streams):
        got.append(step(u, stream=s))
        for _ in range(4):
            busy.append(torch.full((need,), 0xff, dtype=torch.uint8, device="cuda"))
            del busy[:-4]
    torch.cuda.synchronize()
    for u, o, end in zip(users, got, ends):
        assert same(held(u, o), end)


def test_same_result_every_time():
    """No order of arrival enters a result: the same call again, to the last bit."""
    u = batch(seed=3, lens=(3000, 2999, 10, 1))
    c, _, q, wd, _ = u
    a = dar.dar_attn_decode_paged_q4(c, q, wd)
    for _ in range(3):
        assert torch.equal(dar.dar_attn_decode_paged_q4(c, q, wd), a)
