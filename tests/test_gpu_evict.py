"""Eviction of distant tokens by score (dar_cache_evict, dar_cache_evict_paged):
latents, scores, ring and lengths after the call against a plain restatement
in NumPy, value for value (nothing is computed on the values but their
order, so nothing may differ). Slots that the call has no business with hold
marks that must survive it."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

dar = pytest.importorskip("paper_2606_18587_amd")

BF, F32 = torch.bfloat16, torch.float32


def counts(n, w, n_keep):
    """(D, E) of a sequence of n tokens."""
    D = max(n - w, 0)
    over = D - n_keep
    return D, 0 if over <= 0 else (over // w * w if w else over)


def reference(scores, n, w, n_keep, n_fixed):
    """One row: source slot of every slot, and the scores after the call."""
    D, E = counts(n, w, n_keep)
    src, out = np.arange(len(scores)), scores.copy()
    if not E:
        return src, out, 0
    left = D - E
    z = scores[n_fixed:D].astype(np.float64)
    nan = np.isnan(z)
    order = np.lexsort((np.arange(len(z)), -np.where(nan, 0.0, z), nan))
    kept = np.zeros(D, bool)
    kept[:n_fixed] = True
    kept[n_fixed + order[:left - n_fixed]] = True
    src[np.flatnonzero(~kept[:left])] = left + np.flatnonzero(kept[left:])
    out[:left] = scores[src[:left]]
    out[left:n - E] = scores[D:n]
    out[n - E:n] = 0.0
    return src, out, E


def make_scores(kind, shape, g):
    z = np.exp(1.5 * g.standard_normal(shape)).astype(np.float32)
    if kind == "few":       # many ties, zeros among them
        z = np.floor(z)
    elif kind == "same":
        z[:] = 0.25
    elif kind == "odd":     # negative, infinite, NaN, zeros of both signs, subnormal
        odd = np.array([0.0, -0.0, np.inf, -np.inf, np.nan, -np.nan, 1e-42, -1e-42, -1.5, 1.5],
                       np.float32)
        z = np.where(g.random(shape) < 0.5, odd[g.integers(0, len(odd), shape)], z)
    elif kind == "near":    # neighbours in the last bits
        z = (np.float32(1.0).view(np.int32) + g.integers(0, 9, shape).astype(np.int32)).view(np.float32)
    return z


def bits(x):
    x = x.detach().cpu().contiguous()
    return x.view(torch.int16 if x.dtype == BF else torch.int32).numpy()


def same_scores(got, want):
    return np.array_equal(got.detach().cpu().numpy().view(np.int32), want.view(np.int32))


def dense(B, Hkv, dd, w, n, cap, dtype, kind, seed=3):
    g = np.random.Generator(np.random.PCG64(seed))
    c = dar.DarCache(B, Hkv, max(8, dd), dd, w, cap, dtype)
    for t in (c.k_win, c.v_win, c.k_lat, c.v_lat):
        t.copy_(torch.from_numpy(g.standard_normal(tuple(t.shape)).astype(np.float32)))
    c.struct.len = n
    z = make_scores(kind, (B, Hkv, cap), g)
    return c, z


def check_dense(c, z, n_keep, n_fixed, in_place):
    n, w = c.len, c.w
    before = {a: bits(getattr(c, a)).copy() for a in ("k_lat", "v_lat", "k_win", "v_win")}
    s = torch.from_numpy(z).cuda()
    out = s if in_place else torch.full_like(s, 7.0)
    gone = dar.dar_cache_evict(c, s, n_keep, n_fixed=n_fixed, scores_out=None if in_place else out)
    torch.cuda.synchronize()
    for b in range(c.B):
        for g in range(c.Hkv):
            src, want, E = reference(z[b, g], n, w, n_keep, n_fixed)
            assert gone == E and c.len == n - E
            for a in ("k_lat", "v_lat"):
                assert np.array_equal(bits(getattr(c, a)[b, g]), before[a][b, g][src]), (a, b, g)
            assert same_scores(out[b, g, :n], want[:n]), (b, g)
            # entries past the newest token are nobody's
            assert same_scores(out[b, g, n:], z[b, g, n:] if in_place else np.full_like(z[b, g, n:], 7.0))
    if not in_place:
        assert same_scores(s, z)
    for a in ("k_win", "v_win"):
        assert np.array_equal(bits(getattr(c, a)), before[a])
    return gone


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("kind", ["plain", "few", "same", "odd", "near"])
@pytest.mark.parametrize("n,w,n_keep,n_fixed", [
    (700, 32, 400, 4),      # several windows' worth
    (433, 32, 400, 0),      # one token too many: nothing happens (E = 0)
    (464, 32, 400, 0),      # exactly one window's worth
    (5000, 100, 37, 37),    # nearly everything goes; only fixed ones and the remainder stay
    (260, 0, 100, 3),       # no window: E exact
    (90, 1, 0, 0),          # everything distant goes
    (1, 0, 0, 0),           # one token, none stays
    (20, 64, 0, 0),         # nothing distant yet
    (4500, 64, 4000, 3000),
])
def test_dense(n, w, n_keep, n_fixed, kind, in_place):
    c, z = dense(2, 3, 16, w, n, n + 37, BF, kind)
    check_dense(c, z, n_keep, n_fixed, in_place)


@pytest.mark.parametrize("dd,dtype", [(5, BF), (8, BF), (32, BF), (3, F32), (16, F32), (20, F32), (1, BF)])
def test_latent_rows_of_any_size(dd, dtype):
    c, z = dense(1, 2, dd, 16, 1000, 1001, dtype, "few")
    check_dense(c, z, 333, 1, False)


@pytest.mark.parametrize("n,n_keep,kind", [(33333, 20000, "plain"), (70001, 60000, "few"),
                                           (140000, 70000, "plain"), (140000, 300, "same")])
def test_long(n, n_keep, kind):
    c, z = dense(1, 2, 16, 512, n, n, BF, kind)
    assert check_dense(c, z, n_keep, 11, kind == "few") > 0


@pytest.mark.parametrize("B,n", [(15, 12000), (16, 12000), (16, 36000)])
def test_many_rows_with_many_moves(B, n):
    """Dense rows on both sides of the number from which the selecting workgroups make
    long lists of moves themselves, and lists too long for that."""
    c, z = dense(B, 8, 8, 64, n, n, BF, "few")
    assert check_dense(c, z, n // 2, 5, B == 16) > 2048


def test_empty_cache_and_twice():
    c, z = dense(1, 1, 16, 8, 0, 64, BF, "plain")
    assert check_dense(c, z, 0, 0, True) == 0
    c, z = dense(1, 2, 16, 8, 600, 600, BF, "plain")
    assert check_dense(c, z, 300, 0, True) == 288
    s = torch.zeros(1, 2, 600, device="cuda")
    assert dar.dar_cache_evict(c, s, 300) == 0      # already within a window of the budget


class Paged:
    def __init__(self, lens, w, ps, kind="few", Hkv=2, dd=16, dtype=BF, seed=5, holes=()):
        g = np.random.Generator(np.random.PCG64(seed))
        B = len(lens)
        longest = max(max(lens), 1)
        maxb = -(-longest // ps) + 1
        n_pages = B * maxb + 3
        c = dar.DarPagedCache(B, Hkv, max(8, dd), dd, w, ps, maxb, n_pages, dtype)
        for t in (c.k_win, c.v_win, c.k_pool, c.v_pool):
            t.copy_(torch.from_numpy(g.standard_normal(tuple(t.shape)).astype(np.float32)))
        self.bt = g.permutation(n_pages)[:B * maxb].reshape(B, maxb).astype(np.int32)
        for b, blk, entry in holes:
            self.bt[b, blk] = entry
        c.block_table.copy_(torch.from_numpy(self.bt))
        c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        self.c, self.lens, self.z = c, lens, make_scores(kind, (B, Hkv, maxb * ps), g)

    def check(self, n_keep, n_fixed, in_place):
        c, ps, z = self.c, self.c.page_size, self.z
        s = torch.from_numpy(z).cuda()
        out = s if in_place else torch.full_like(s, 7.0)
        names = ("k_pool", "v_pool")
        old = {a: bits(getattr(c, a)).copy() for a in names}
        want = {a: x.copy() for a, x in old.items()}
        rings = [bits(x).copy() for x in (c.k_win, c.v_win)]
        dar.dar_cache_evict_paged(c, s, n_keep, n_fixed=n_fixed, scores_out=None if in_place else out)
        torch.cuda.synchronize()
        lens = []
        for b, n in enumerate(self.lens):
            live = 1 <= n <= c.cap
            E = 0
            for g in range(c.Hkv):
                base = z[b, g] if in_place else np.full_like(z[b, g], 7.0)
                if live:
                    src, after, E = reference(z[b, g], n, c.w, n_keep, n_fixed)
                    base = np.concatenate([after[:n], base[n:]])
                    for e in np.flatnonzero(src != np.arange(len(src))):
                        to, fr = self.bt[b, e // ps], self.bt[b, src[e] // ps]
                        for a in names:
                            if 0 <= to < c.n_pages:
                                row = old[a][fr, g, src[e] % ps] if 0 <= fr < c.n_pages else 0
                                want[a][to, g, e % ps] = row
                assert same_scores(out[b, g], base), (b, g)
            lens.append(n - E)
        assert c.lens.cpu().tolist() == lens
        for a in names:
            assert np.array_equal(bits(getattr(c, a)), want[a]), a
        for x, y in zip((c.k_win, c.v_win), rings):
            assert np.array_equal(bits(x), y)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("lens,w,ps,n_keep,n_fixed", [
    ([700, 1, 0, 64, 333, 1200], 32, 64, 200, 4),
    ([700, 1, 65, -701, 333, 2500], 0, 32, 128, 64),   # one sequence overflowed, no window
    ([5000, 4000, 130], 100, 256, 1000, 512),
])
def test_paged(lens, w, ps, n_keep, n_fixed, in_place):
    Paged(lens, w, ps).check(n_keep, n_fixed, in_place)


def test_paged_odd_scores_and_unmapped_pages():
    """Entries outside the pool: what is moved from there reads as zeros, what
    goes there is dropped."""
    Paged([900, 640], 16, 32, kind="odd", holes=[(0, 0, -1), (0, 20, 9999), (1, 3, -5), (1, 18, 1 << 30)]
          ).check(300, 0, True)


def test_paged_lens_beyond_capacity_left_alone():
    p = Paged([300, 400], 16, 64)
    p.lens = [300, 10 ** 6]
    p.c.lens.copy_(torch.tensor(p.lens, dtype=torch.int32))
    p.check(100, 0, True)


def test_many_rows():
    """More rows than compute units."""
    c, z = dense(40, 8, 16, 8, 200, 200, BF, "few")
    check_dense(c, z, 100, 0, True)


@pytest.mark.parametrize("n,n_keep,n_fixed,kind", [
    (8192 + 16, 5000, 0, "few"), (8192 + 19, 5000, 3, "same"), (8192 + 20, 5000, 3, "near"),   # keys held: border
    (34816 + 16, 30000, 0, "plain"), (34816 + 17, 17000, 0, "near"), (34816 + 19, 100, 2, "odd"),
    (70000, 69000, 0, "same"), (140001, 66000, 5, "odd"), (140001, 139000, 131072, "few")])
def test_row_lengths_at_the_kernels_borders(n, n_keep, n_fixed, kind):
    c, z = dense(1, 2, 16, 16, n, n + n % 4, BF, kind)
    check_dense(c, z, n_keep, n_fixed, n % 2 == 0)


def test_many_rows_many_moves():
    """Enough rows that the selecting workgroups make the moves, thousands each."""
    c, z = dense(16, 8, 16, 16, 9000, 9000, BF, "few")
    check_dense(c, z, 4500, 7, False)
    c, z = dense(16, 8, 8, 16, 36000, 36000, BF, "plain")
    check_dense(c, z, 28000, 0, True)
    Paged([9000 - 71 * b for b in range(64)], 16, 64, kind="near").check(3000, 64, True)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("kind", ["plain", "few", "same", "odd"])
@pytest.mark.parametrize("w,ps,n_keep,n_fixed", [(48, 64, 20000, 129), (0, 256, 300, 300), (7, 32, 0, 0)])
def test_long_and_short_sequences(w, ps, n_keep, n_fixed, kind, in_place):
    """Several workgroups a row: rows that end in any of them, that lose nothing, that
    are empty; ties that are cut off inside a share."""
    Paged([61234, 1, 0, 36001, 20048, 20055, -3, 20100, 130], w, ps, kind, Hkv=1).check(
        n_keep, n_fixed, in_place)


@pytest.mark.parametrize("n_keep", [60000, 36000, 40])
def test_long_rows_odd_capacity(n_keep):
    """A capacity that aligns no row but the first; nothing to evict among them."""
    for n in (40000, 44443):
        c, z = dense(3, 1, 16, 32, n, 44443, BF, "few")
        check_dense(c, z, n_keep, 39, False)
