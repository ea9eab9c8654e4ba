"""The 4-bit latent format and a decode step over it, restated in fp64 from their
definitions (include/dar_q4.h, Eq. 2-4), for the tests of the 4-bit cache."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def groups(dd):
    return [slice(c, min(c + 32, dd)) for c in range(0, dd, 32)]


def quantise(x):
    """Rows x [n, dd] (fp64 values): codes [n, 4 ceil(dd / 8)] and scale bytes
    [n, ceil(dd / 32)], uint8."""
    n, dd = x.shape
    nib = np.zeros((n, 8 * -(-dd // 8)), np.uint8)
    exps = np.zeros((n, len(groups(dd))), np.uint8)
    for j, cols in enumerate(groups(dd)):
        y = x[:, cols]
        bad = ~np.isfinite(y).all(1)
        y = np.where(bad[:, None], 0.0, y)
        a = np.abs(y).max(1)
        e = np.full(n, -124)
        for k in range(-124, 126):            # the smallest power of two with a <= 7 s
            e = np.where(a > 7 * 2.0 ** e, k, e)
        e = np.clip(np.where(a > 7 * 2.0 ** e, 125, e), -124, 125)
        r = np.abs(y) / 2.0 ** e[:, None]
        dist = np.abs(r[:, :, None] - LEVELS)
        even = np.arange(8) % 2               # of two equal distances the even index
        order = np.lexsort((np.broadcast_to(even, dist.shape), dist), axis=-1)
        code = order[:, :, 0].astype(np.uint8) | (np.signbit(y).astype(np.uint8) << 3)
        nib[:, cols] = np.where(bad[:, None], 0, code)
        exps[:, j] = np.where(bad, 255, e + 127)
    return nib[:, 0::2] | (nib[:, 1::2] << 4), exps


def values(codes, exps, dd):
    """The rows [n, dd] that codes and scale bytes stand for."""
    nib = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], 2 * codes.shape[1])[:, :dd]
    s = np.where(exps == 255, np.nan, 2.0 ** (exps.astype(np.float64) - 127))
    v = np.where(nib >= 8, -1.0, 1.0) * LEVELS[nib & 7]
    return v * np.repeat(s, 32, axis=1)[:, :dd]


def decode(q, k_lat, v_lat, k_win, v_win, wu, n, w):
    """One sequence and KV head: q [G,d]; latents [>= n - w, dd] by slot, rings
    [>= w,d], wu [dd,d]. Returns o [G,d], sum of p |v| [G,d] and, per query head, the
    largest sum of absolute terms of a score [G,1]."""
    d = q.shape[1]
    far = max(n - w, 0)
    ring = np.arange(far, n) % max(w, 1)
    qt = q @ wu.T                              # absorbed queries
    s = np.concatenate([qt @ k_lat[:far].T, q @ k_win[ring].T], 1) / np.sqrt(d)
    p = np.exp(s - s.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    o = (p[:, :far] @ v_lat[:far]) @ wu + p[:, far:] @ v_win[ring]
    mass = (p[:, :far] @ np.abs(v_lat[:far])) @ np.abs(wu) + p[:, far:] @ np.abs(v_win[ring])
    aq = np.abs(q) @ np.abs(wu).T
    terms = np.concatenate([aq @ np.abs(k_lat[:far]).T, np.abs(q) @ np.abs(k_win[ring]).T], 1)
    return o, mass, terms.max(1, keepdims=True) / np.sqrt(d)


def decode_atol(o, mass, terms, n, d, dd, bf16):
    """How far an output may be off.
    Scores: chains of at most d + dd + 8 fp32 operations, each off by 2^-24 of the
    sum of absolute terms; in bf16 the absorbed query is a pair of bf16, which
    leaves 2^-16 of every element. A score off by e changes a weight by the factor
    exp(e) and the denominator by as much. Weights: the exponential, the scale to
    the running reference and to the joined one, a few 2^-23 each; in bf16 a
    pair of bf16 again, 2^-16. Sums of weights and values: at most n + dd + 64
    operations. Then the output's own rounding, half a step."""
    score = (d + dd + 8) * 2.0 ** -24 * terms + (2.0 ** -16 * terms if bf16 else 0.0)
    weight = 2 * np.expm1(score) + 16 * 2.0 ** -23 + (2.0 ** -16 if bf16 else 0.0)
    return (weight + 2 * (n + dd + 64) * 2.0 ** -24) * mass + (2.0 ** -8 if bf16 else 2.0 ** -24) * np.abs(o) + 1e-37
