"""Decode steps that score the cached tokens (dar_attn_decode_scored,
dar_attn_decode_paged_scored) and decode steps over a shared prefix
(dar_attn_decode_paged_prefix) against the fp64 restatement of
serving_ref.py: outputs within the tolerance of the decode tests (2e-2 for
bf16, 1e-4 for fp32, on unit-scale values), scores within the fp32 rounding
that weight_rtol derives."""
import numpy as np
import pytest
import torch

from tests.dev import tol
from tests.serving_ref import f64, step, weight_rtol

pytestmark = pytest.mark.gpu

dar = pytest.importorskip("paper_2606_18587_amd")

BF, F32 = torch.bfloat16, torch.float32


def rand(g, *shape, dtype=BF, std=1.0):
    return (torch.randn(*shape, generator=g) * std).to(dtype).cuda()


def weights(g, Hkv, d, dd, untied, dtype=BF):
    wd = rand(g, Hkv, d, dd, dtype=dtype, std=d ** -0.5)
    wu = rand(g, Hkv, dd, d, dtype=dtype, std=dd ** -0.5) if untied else None
    return wd, wu, f64(wd).transpose(0, 2, 1) if wu is None else f64(wu)


def check_scores(got, old, p, n, first, rtol):
    """got, old: a row's entries; p [G,n] the reference weights."""
    want = old.astype(np.float64)
    want[first:n] += p[:, first:].sum(0)
    err = np.abs(got - want)
    room = np.zeros_like(want)
    room[first:n] = p[:, first:].sum(0) * rtol + 2.0 ** -24 * np.abs(want[first:n])
    assert (err <= room).all(), (err - room).max()


class Dense:
    def __init__(self, B, Hq, Hkv, d, dd, w, n, cap, dtype=BF, untied=False, seed=1, qstd=2.0):
        g = torch.Generator().manual_seed(seed)
        self.c = c = dar.DarCache(B, Hkv, d, dd, w, cap, dtype)
        for t in (c.k_win, c.v_win, c.k_lat, c.v_lat):
            t.copy_(torch.randn(t.shape, generator=g))
        c.struct.len = n
        # slots past the distant tokens are not read
        c.k_lat[:, :, max(n - w, 0):] = float("nan")
        c.v_lat[:, :, max(n - w, 0):] = float("nan")
        self.q = rand(g, B, Hq, d, dtype=dtype, std=qstd)
        self.wd, self.wu, self.up = weights(g, Hkv, d, dd, untied, dtype)
        self.old = torch.rand(B, Hkv, cap, generator=g).cuda()
        self.B, self.G, self.dtype = B, Hq // Hkv, dtype

    def check(self, in_place=False):
        c, n = self.c, self.c.len
        sc = self.old.clone()
        out = sc if in_place else torch.full_like(sc, 9.0)
        o = dar.dar_attn_decode_scored(c, self.q, self.wd, sc, self.wu,
                                       scores_out=None if in_place else out)
        torch.cuda.synchronize()
        k_lat, v_lat, k_win, v_win, q = (f64(x) for x in (c.k_lat, c.v_lat, c.k_win, c.v_win, self.q))
        old, got, o = self.old.cpu().numpy(), out.cpu().numpy(), f64(o)
        for b in range(self.B):
            for g in range(c.Hkv):
                hs = slice(g * self.G, (g + 1) * self.G)
                ro, p, terms = step(q[b, hs], k_lat[b, g], v_lat[b, g], k_win[b, g], v_win[b, g],
                                    self.up[g], n, c.w)
                assert np.abs(o[b, hs] - ro).max() <= tol("bf16" if self.dtype == BF else "f32")
                check_scores(got[b, g, :n], old[b, g, :n], p, n, 0, weight_rtol(terms, c.d, c.d_down))
                rest = old[b, g, n:] if in_place else np.full_like(old[b, g, n:], 9.0)
                assert np.array_equal(got[b, g, n:], rest)
        return o


@pytest.mark.parametrize("d,dd,G", [(64, 16, 1), (64, 32, 2), (128, 16, 4), (128, 32, 8), (64, 16, 8)])
@pytest.mark.parametrize("w,n", [(32, 1), (32, 32), (32, 33), (48, 500), (0, 333), (1, 97), (700, 650)])
def test_dense_bf16(d, dd, G, w, n):
    Dense(2, 3 * G, 3, d, dd, w, n, n + 5, untied=n % 2 == 1).check(in_place=w == 48)


def test_dense_long_split_and_whole():
    Dense(1, 8, 2, 64, 16, 256, 20011, 20011).check()            # several records a head
    Dense(40, 16, 8, 64, 16, 32, 300, 300, seed=2).check()      # one each


@pytest.mark.parametrize("dtype,d,dd,w,n,G", [(F32, 64, 16, 32, 700, 4), (F32, 80, 20, 7, 131, 8),
                                              (F32, 16, 3, 0, 50, 1), (BF, 96, 24, 40, 300, 2),
                                              (F32, 256, 256, 5, 40, 1), (F32, 64, 16, 300, 5000, 2),
                                              (F32, 7, 7, 4, 9, 1)])
def test_dense_other_shapes(dtype, d, dd, w, n, G):
    Dense(2, 2 * G, 2, d, dd, w, n, n + 1, dtype=dtype, untied=d == 80).check(in_place=d == 16)


def test_peaked_scores():
    """Queries whose scores spread over hundreds: weights from 1 down to 0."""
    Dense(1, 4, 2, 64, 16, 32, 600, 600, qstd=60.0).check()


class Paged:
    """Sequences over one pool; the first n_prefix tokens of all of them in the
    pages of `blocks`."""

    def __init__(self, lens, Hq, Hkv, d, dd, w, ps, n_prefix=0, untied=False, seed=3, unmapped=()):
        g = torch.Generator().manual_seed(seed)
        B = len(lens)
        shared = n_prefix // ps
        maxb = max(-(-max(max(lens), 1) // ps), shared) + 1
        own = maxb - shared
        n_pages = shared + B * own + 2
        self.c = c = dar.DarPagedCache(B, Hkv, d, dd, w, ps, maxb, n_pages, BF)
        for t in (c.k_win, c.v_win, c.k_pool, c.v_pool):
            t.copy_(torch.randn(t.shape, generator=g))
        perm = torch.randperm(n_pages, generator=g)
        bt = torch.cat([perm[:shared].expand(B, shared), perm[shared:shared + B * own].reshape(B, own)], 1)
        bt = bt.to(torch.int32).contiguous()
        for b, blk, entry in unmapped:
            if b is None:
                bt[:, blk] = entry
            else:
                bt[b, blk] = entry
        self.bt = bt.numpy()
        c.block_table.copy_(bt)
        c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        self.blocks = bt[0, :shared].contiguous().cuda() if shared else None
        self.q = rand(g, B, Hq, d, std=2.0)
        self.wd, self.wu, self.up = weights(g, Hkv, d, dd, untied)
        self.old = torch.rand(B, Hkv, maxb * ps, generator=g).cuda()
        self.lens, self.n_prefix, self.G = lens, n_prefix, Hq // Hkv

    def poison(self):
        """NaN in every slot of pool and ring that no sequence's tokens fill."""
        filled = torch.zeros(self.c.n_pages, self.c.page_size, dtype=torch.bool)
        for b, n in enumerate(self.lens):
            slots = torch.arange(max(n - self.c.w, 0))
            filled[torch.from_numpy(self.bt[b]).long()[slots // self.c.page_size], slots % self.c.page_size] = True
            self.c.k_win[b, :, max(n, 0):] = float("nan")
            self.c.v_win[b, :, max(n, 0):] = float("nan")
        for pool in (self.c.k_pool, self.c.v_pool):
            pool.masked_fill_(~filled.cuda()[:, None, :, None], float("nan"))
        return self

    def rows(self, pool, b, g):
        """Latents of sequence b in slot order."""
        ok = (self.bt[b] >= 0) & (self.bt[b] < self.c.n_pages)
        x = pool[np.where(ok, self.bt[b], 0), g] * ok[:, None, None]
        return x.reshape(-1, x.shape[2])

    def check(self, scored, in_place=True):
        c, first = self.c, self.n_prefix
        sc = self.old.clone()
        out = sc if in_place else torch.full_like(sc, 9.0)
        if scored:
            o = dar.dar_attn_decode_paged_scored(c, self.q, self.wd, sc, self.wu,
                                                 prefix_blocks=self.blocks,
                                                 scores_out=None if in_place else out)
        else:
            blocks = torch.empty(0, dtype=torch.int32, device="cuda") if self.blocks is None else self.blocks
            o = dar.dar_attn_decode_paged_prefix(c, self.q, self.wd, blocks, self.wu)
        torch.cuda.synchronize()
        kp, vp, k_win, v_win, q = (f64(x) for x in (c.k_pool, c.v_pool, c.k_win, c.v_win, self.q))
        old, got, o = self.old.cpu().numpy(), out.cpu().numpy(), f64(o)
        for b, n in enumerate(self.lens):
            if n < 1:
                assert np.isnan(o[b]).all()
                n = 0
            for g in range(c.Hkv):
                untouched = old[b, g].copy() if in_place else np.full_like(old[b, g], 9.0)
                if n:
                    hs = slice(g * self.G, (g + 1) * self.G)
                    ro, p, terms = step(q[b, hs], self.rows(kp, b, g), self.rows(vp, b, g), k_win[b, g],
                                        v_win[b, g], self.up[g], n, c.w)
                    assert np.abs(o[b, hs] - ro).max() <= tol("bf16"), (b, g)
                    if scored:
                        check_scores(got[b, g, first:n], old[b, g, first:n], p[:, first:], n - first, 0,
                                     weight_rtol(terms, c.d, c.d_down)) if n > first else None
                        untouched[first:n] = got[b, g, first:n]
                if scored:
                    assert np.array_equal(got[b, g], untouched), (b, g)
        return o


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("d,dd,Hq,Hkv", [(64, 16, 8, 2), (64, 32, 2, 2), (128, 16, 8, 1), (128, 32, 6, 3)])
def test_paged_scored(d, dd, Hq, Hkv, in_place):
    Paged([1, 37, 0, 300, 64, -12, 511, 129], Hq, Hkv, d, dd, 32, 64, untied=d == 128).check(True, in_place)


@pytest.mark.parametrize("w,ps", [(0, 32), (1, 256), (600, 64)])
def test_paged_scored_windows(w, ps):
    Paged([1, 300, 64, 4000], 8, 2, 64, 16, w, ps).check(True)


@pytest.mark.parametrize("scored", [False, True])
@pytest.mark.parametrize("d,dd,Hq,Hkv,w,ps,n_prefix", [
    (64, 16, 8, 2, 32, 64, 512), (64, 32, 3, 3, 100, 32, 96), (128, 16, 8, 1, 0, 256, 256),
    (128, 32, 8, 4, 300, 64, 1024), (64, 16, 4, 2, 16, 64, 8192)])
def test_prefix(d, dd, Hq, Hkv, w, ps, n_prefix, scored):
    """Sequences that end inside the prefix, at its end, with the prefix's end in
    their window, just and far past it; empty and overflowed ones."""
    lens = [n_prefix + x for x in (0, 1, w, w + 1, w + 777)] + [
        0, -9, 1, n_prefix // 2, max(n_prefix + w - 1, 1), n_prefix + 2 * w + 33]
    Paged(lens, Hq, Hkv, d, dd, w, ps, n_prefix, untied=d == 64).check(scored)


@pytest.mark.parametrize("scored", [False, True])
@pytest.mark.parametrize("B,Hq,Hkv", [(1, 1, 1), (9, 8, 2), (70, 4, 1), (130, 2, 2)])
def test_prefix_batches(B, Hq, Hkv, scored):
    """Row tiles that are full, broken and single; batches past the 64 sequences
    that a wavefront plans by itself."""
    Paged([640 + 40 + 13 * (b % 11) for b in range(B)], Hq, Hkv, 64, 16, 40, 64, 640).check(scored)


@pytest.mark.parametrize("scored", [False, True])
@pytest.mark.parametrize("n_prefix", [0, 128])
@pytest.mark.parametrize("B", [256, 257, 300, 512, 513])
def test_batches_past_a_workgroups_threads(B, n_prefix, scored):
    """More sequences than the workgroup that plans them has threads: empty and
    overflowed ones, one part and several, in no order."""
    g = torch.Generator().manual_seed(B)
    kinds = torch.tensor([0, -3, 1, 40, 200, 700, 1100])
    lens = kinds[torch.randint(len(kinds), (B,), generator=g)]
    lens = torch.where(lens > 0, lens + torch.randint(0, 90, (B,), generator=g), lens).tolist()
    lens[-1] = 1177
    Paged(lens, 4, 2, 64, 16, 40, 64, n_prefix, seed=B).check(scored)


@pytest.mark.parametrize("scored", [False, True])
def test_lengths_past_a_capacity_that_is_all_prefix(scored):
    """No window and a prefix of the whole capacity: no sequence has a part of its
    own, also where its length is past the capacity (it then counts as that).
    The workspace holds no count that could be read."""
    p = Paged([128, 100, 128, 128], 8, 2, 64, 16, 0, 32, 128)
    c = p.c
    c.block_table = c.block_table[:, :4].contiguous()
    c.max_blocks = 4
    c.lens.copy_(torch.tensor([133, 100, 160, 1 << 30], dtype=torch.int32))
    need = dar.dar_decode_prefix_workspace_bytes(dar.make_shape(4, 8, 2, 64, 16, 0, BF), 128, 128)
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
    sc = p.old[:, :, :128].contiguous()
    kept = sc.clone()
    if scored:
        o = dar.dar_attn_decode_paged_scored(c, p.q, p.wd, sc, prefix_blocks=p.blocks, ws=ws)
    else:
        o = dar.dar_attn_decode_paged_prefix(c, p.q, p.wd, p.blocks, ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(sc, kept)
    kp, vp, q, o = (f64(x) for x in (c.k_pool, c.v_pool, p.q, o))
    for b, n in enumerate(p.lens):
        for g in range(2):
            ro, _, _ = step(q[b, 4 * g:4 * g + 4], p.rows(kp, b, g), p.rows(vp, b, g), np.zeros((1, 64)),
                            np.zeros((1, 64)), p.up[g], n, 0)
            assert np.abs(o[b, 4 * g:4 * g + 4] - ro).max() <= tol("bf16"), (b, g)


@pytest.mark.parametrize("scored", [False, True])
def test_prefix_none_and_unmapped_pages(scored):
    Paged([5, 300, 64], 4, 2, 64, 16, 32, 64).check(scored)
    Paged([900, 700], 4, 2, 64, 16, 32, 64, 512,
          unmapped=[(None, 3, -1), (None, 0, 1 << 30), (0, 10, -7)]).check(scored)


@pytest.mark.parametrize("scored", [False, True])
def test_long_prefix_of_a_batch(scored):
    """Runs of many passes, one row tile broken."""
    Paged([16384 + 50 + 97 * b for b in range(36)], 8, 1, 64, 16, 40, 64, 16384).check(scored)


@pytest.mark.parametrize("scored", [False, True])
@pytest.mark.parametrize("d,dd,w,n_prefix", [(64, 16, 100, 512), (128, 32, 37, 128), (64, 32, 200, 64),
                                             (128, 16, 64, 0)])
def test_unfilled_slots_are_not_read(d, dd, w, n_prefix, scored):
    """As after the prompt and a few steps: the prefix's last tokens are still in the
    windows, and pages and rings end in memory that nothing wrote."""
    Paged([n_prefix + x for x in (3, 1, 9, 2)], 8, 2, d, dd, w, 64, n_prefix).poison().check(scored)
    Paged([n_prefix + x for x in (70, 5, 0, 333)], 4, 2, d, dd, w, 32, n_prefix).poison().check(scored)


@pytest.mark.parametrize("dtype,d,dd", [(BF, 64, 16), (BF, 128, 32), (F32, 64, 16), (BF, 96, 24)])
@pytest.mark.parametrize("n", [1, 40, 130])
def test_unfilled_ring_is_not_read(dtype, d, dd, n):
    c = Dense(2, 8, 2, d, dd, 130, n, 200, dtype=dtype)
    c.c.k_win[:, :, n:] = float("nan")
    c.c.v_win[:, :, n:] = float("nan")
    c.check()


def test_prefix_blocks_stand_for_the_first_blocks():
    """The block table's entries for the prefix are not read: they may be unset."""
    p = Paged([700 + 31 * b for b in range(5)], 8, 2, 64, 16, 32, 64, 512)
    want = p.check(False)
    p.c.block_table[:, :8] = -1
    got = f64(dar.dar_attn_decode_paged_prefix(p.c, p.q, p.wd, p.blocks))
    assert np.abs(got - want).max() <= 2 * tol("bf16")


def test_prefix_matches_paged_decode():
    """The same cache through the decode that reads every sequence's own pages:
    each is within its tolerance of the definition."""
    p = Paged([2048 + 70 + 31 * b for b in range(12)], 16, 4, 64, 16, 64, 64, 2048)
    a = p.check(False)
    b = f64(dar.dar_attn_decode_paged(p.c, p.q, p.wd))
    assert np.abs(a - b).max() <= 2 * tol("bf16")


def test_order_does_not_change_results():
    p = Paged([2048 + 70 + 331 * b for b in range(12)], 16, 4, 64, 16, 64, 64, 2048)
    first, one = None, None
    for _ in range(3):
        sc = p.old.clone()
        o = dar.dar_attn_decode_paged_scored(p.c, p.q, p.wd, sc, prefix_blocks=p.blocks)
        torch.cuda.synchronize()
        if first is None:
            first, one = o, sc
        assert torch.equal(o.view(torch.int16), first.view(torch.int16)) and torch.equal(sc, one)
