"""How exact the outputs of the serving decodes are (bf16, matrix cores): scores,
sums and the merge in fp32, weights of 16 bits against the values, one rounding
of the result."""
import numpy as np
import pytest
import torch

from tests.serving_ref import f64, step, weight_rtol
from tests.test_gpu_scored import BF, Dense, Paged

pytestmark = pytest.mark.gpu

dar = pytest.importorskip("paper_2606_18587_amd")


def room(p, values, want, terms, d, dd):
    """p [G,n], values [n,d] the absolute terms of the lifted values: how far an
    element of the output may be off. A weight is off by weight_rtol of itself;
    it meets the values as two bf16 operands, whose roundings (2^-8 each at most)
    leave 2^-16 of it; the n products and the d_down terms of the lift are added
    up in fp32; then the result is rounded to bf16, by 2^-8 of itself at most."""
    n = p.shape[1]
    sums = (2.0 ** -16 + weight_rtol(terms, d, dd) + (n + dd + 8) * 2.0 ** -24) * (p @ values)
    return sums + 2.0 ** -8 * (np.abs(want) + sums)


def check_rows(o, q, k_lat, v_lat, k_win, v_win, up, n, w):
    d, dd = q.shape[1], up.shape[0]
    want, p, terms = step(q, k_lat, v_lat, k_win, v_win, up, n, w)
    far = max(n - w, 0)
    values = np.concatenate([np.abs(v_lat[:far]) @ np.abs(up), np.abs(v_win[np.arange(far, n) % max(w, 1)])])
    off = np.abs(o - want) - room(p, values, want, terms, d, dd)
    assert (off <= 0).all(), (off.max(), n)


@pytest.mark.parametrize("d,dd,G", [(64, 16, 4), (64, 32, 8), (128, 16, 1), (128, 32, 2)])
@pytest.mark.parametrize("w,n", [(32, 1), (32, 5), (0, 3), (40, 300), (100, 2000)])
def test_dense(d, dd, G, w, n):
    x = Dense(3, 2 * G, 2, d, dd, w, n, n + 3, untied=n == 300, seed=d + n)
    c = x.c
    o = f64(dar.dar_attn_decode_scored(c, x.q, x.wd, x.old, x.wu))
    k_lat, v_lat, k_win, v_win, q = (f64(t) for t in (c.k_lat, c.v_lat, c.k_win, c.v_win, x.q))
    for b in range(3):
        for g in range(2):
            hs = slice(g * G, g * G + G)
            check_rows(o[b, hs], q[b, hs], k_lat[b, g], v_lat[b, g], k_win[b, g], v_win[b, g], x.up[g], n, w)


@pytest.mark.parametrize("d,dd,Hq,Hkv,w,n_prefix", [(64, 16, 8, 2, 32, 0), (64, 32, 8, 1, 40, 512),
                                                    (128, 32, 4, 2, 64, 256), (128, 16, 2, 2, 0, 1024),
                                                    (64, 16, 8, 2, 16, 2048)])
def test_paged_with_and_without_scores(d, dd, Hq, Hkv, w, n_prefix):
    """The two forms of a step give the same outputs to the last bit."""
    x = Paged([n_prefix + n for n in (1, 3, 50, 200, 900)], Hq, Hkv, d, dd, w, 64, n_prefix, untied=dd == 32)
    c, G = x.c, Hq // Hkv
    a = dar.dar_attn_decode_paged_scored(c, x.q, x.wd, x.old, x.wu, prefix_blocks=x.blocks)
    blocks = torch.empty(0, dtype=torch.int32, device="cuda") if x.blocks is None else x.blocks
    b = dar.dar_attn_decode_paged_prefix(c, x.q, x.wd, blocks, x.wu)
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    kp, vp, k_win, v_win, q, o = (f64(t) for t in (c.k_pool, c.v_pool, c.k_win, c.v_win, x.q, a))
    for b, n in enumerate(x.lens):
        for g in range(Hkv):
            hs = slice(g * G, g * G + G)
            check_rows(o[b, hs], q[b, hs], x.rows(kp, b, g), x.rows(vp, b, g), k_win[b, g], v_win[b, g],
                       x.up[g], n, w)


@pytest.mark.parametrize("d,dd,G", [(64, 16, 4), (128, 32, 8)])
def test_one_token_is_its_value(d, dd, G):
    """One token has weight 1: the output is its value, as dar_attn_decode gives it."""
    x = Dense(16, 4 * G, 4, d, dd, 32, 1, 8, seed=d)
    want = x.c.v_win[:, :, 0].repeat_interleave(G, 1)
    assert torch.equal(dar.dar_attn_decode(x.c, x.q, x.wd), want)
    assert torch.equal(dar.dar_attn_decode_scored(x.c, x.q, x.wd, x.old), want)
    y = Paged([1] * 16, 4 * G, 4, d, dd, 32, 64)
    want = y.c.v_win[:, :, 0].repeat_interleave(G, 1)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert torch.equal(dar.dar_attn_decode_paged_prefix(y.c, y.q, y.wd, none), want)
    assert torch.equal(dar.dar_attn_decode_paged_scored(y.c, y.q, y.wd, y.old), want)
