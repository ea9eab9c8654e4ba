"""A paged cache whose latents of one head pass 2^32 bytes: a few tokens far apart
hold all the weight, the others have zero latents, so that the definition is
short to write down and a token read from the wrong place shows. (Dense
decodes take at most 2^26 bytes of latents a head.)"""
import numpy as np
import pytest
import torch

from tests.dev import tol
from tests.serving_ref import f64, weight_rtol

pytestmark = pytest.mark.gpu

dar = pytest.importorskip("paper_2606_18587_amd")

BF = torch.bfloat16
D, DD, W, G = 64, 32, 64, 4
N = (1 << 26) + 5000   # tokens: 2^26 latents of 32 bf16 are 2^32 bytes
FAR = N - W
AT = [5, (1 << 24) + 3, (1 << 25) + 77, (1 << 26) - 1, (1 << 26) + 4000, FAR - 1]


def planted(k_lat, v_lat, k_win, v_win):
    """Latent rows [tokens, DD] of one head and rings [W, D], filled in; the query,
    the weights and the step's output and weights by the definition: those of the
    tokens AT, of one token with zero latents, and of the window by position."""
    g = torch.Generator().manual_seed(9)
    wd = (torch.randn(1, D, DD, generator=g) * D ** -0.5).to(BF)
    up = f64(wd)[0].T
    q = (torch.randn(1, 1, D, generator=g) * 2 + torch.randn(1, G, D, generator=g) * 0.2).to(BF)
    mean = f64(q)[0].mean(0) @ up.T / np.sqrt(D)
    want = 25.0 + np.random.default_rng(9).random(len(AT))
    rows = torch.from_numpy(mean[None] / (mean @ mean) * want[:, None]).to(BF)
    vals = (torch.randn(len(AT), DD, generator=g) * 3).to(BF)
    k_lat[AT], v_lat[AT] = rows.cuda(), vals.cuda()
    for t in (k_win, v_win):
        t.copy_(torch.randn(W, D, generator=g))
    qf, ring = f64(q)[0], np.arange(FAR, N) % W
    keys = np.concatenate([f64(rows) @ up, f64(k_win)[ring]])
    s = qf @ keys.T / np.sqrt(D)
    total = np.exp(s).sum(1) + (FAR - len(AT))
    p = np.exp(s) / total[:, None]
    o = p @ np.concatenate([f64(vals) @ up, f64(v_win)[ring]])
    a = np.concatenate([np.abs(f64(rows)) @ np.abs(up), np.abs(f64(k_win)[ring])])
    terms = (np.abs(qf) @ a.T / np.sqrt(D)).max()
    return q.cuda(), wd.cuda(), o, p.sum(0), (1 / total).sum(), terms


def check(o, scores, want, p, rest, terms):
    assert np.abs(f64(o)[0] - want).max() <= tol("bf16")
    rtol = weight_rtol(terms, D, DD)
    got = scores[0, 0]
    at = AT + list(range(FAR, N))
    assert (np.abs(f64(got[at]) - p) <= rtol * p).all()
    others = f64(got[[0, 6, (1 << 24) + 4, (1 << 25) - 1, 1 << 25, 1 << 26, FAR - 2]])
    assert (np.abs(others - rest) <= rtol * rest).all()
    assert (got[N:] == 0).all()


def test_paged():
    """Pages of 2^24 tokens, in no order; with and without scores, and the plain paged
    decode."""
    page, order = 1 << 24, [3, 0, 4, 1, 2]
    c = dar.DarPagedCache(1, 1, D, DD, W, page, 5, 5, BF)
    c.block_table.copy_(torch.tensor([order], dtype=torch.int32))
    c.lens.fill_(N)
    k_lat, v_lat = (torch.zeros(5 * page, DD, dtype=BF, device="cuda") for _ in range(2))
    q, wd, want, p, rest, terms = planted(k_lat, v_lat, c.k_win[0, 0], c.v_win[0, 0])
    for pool, lat in ((c.k_pool, k_lat), (c.v_pool, v_lat)):
        for i, at in enumerate(order):
            pool[at, 0] = lat[i * page:(i + 1) * page]
    del k_lat, v_lat, lat
    scores = torch.zeros(1, 1, 5 * page, device="cuda")
    o = dar.dar_attn_decode_paged_scored(c, q, wd, scores)
    check(o, scores, want, p, rest, terms)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert np.abs(f64(dar.dar_attn_decode_paged_prefix(c, q, wd, none))[0] - want).max() <= tol("bf16")
    assert np.abs(f64(dar.dar_attn_decode_paged(c, q, wd))[0] - want).max() <= tol("bf16")
    # half of it as a prefix
    blocks = c.block_table[0, :2].contiguous()
    o = dar.dar_attn_decode_paged_scored(c, q, wd, scores.zero_(), prefix_blocks=blocks)
    assert np.abs(f64(o)[0] - want).max() <= tol("bf16")
    assert (scores[0, 0, :2 * page] == 0).all()
