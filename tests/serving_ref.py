"""A decode step restated in fp64 from the contents of a cache (Eq. 2-4: distant
tokens lifted to full dimension, one softmax over both regions), for the tests
of the serving operators."""
import numpy as np


def f64(x):
    return x.detach().double().cpu().numpy()


def step(q, k_lat, v_lat, k_win, v_win, wu, n, w):
    """One sequence and KV head: q [G,d], latents [>= n - w, dd] by slot, rings
    [w,d], wu [dd,d]. Returns o [G,d], weights [G,n], and the largest sum of
    absolute terms of a score (natural-log units)."""
    d = q.shape[1]
    far = max(n - w, 0)
    ring = np.arange(far, n) % max(w, 1)
    k = np.concatenate([k_lat[:far] @ wu, k_win[ring]])
    v = np.concatenate([v_lat[:far] @ wu, v_win[ring]])
    s = q @ k.T / np.sqrt(d)
    p = np.exp(s - s.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    a = np.concatenate([np.abs(k_lat[:far]) @ np.abs(wu), np.abs(k_win[ring])])
    terms = (np.abs(q) @ a.T / np.sqrt(d)).max() if n else 0.0
    return p @ v, p, terms


def weight_rtol(terms, d, dd):
    """How far a weight may be off, relative to itself, when scores and denominator
    are computed in fp32: a score is a chain of at most d + 3 dd + 4 fp32
    additions of terms whose absolute values add up to `terms`, each rounded by
    2^-24 at most (the operands' three bf16 parts leave 2^-24 of each), and the
    denominator's logarithm is off by as much; the exponentials and the
    additions after them round by 2^-23 a few times over."""
    return 2 * (d + 3 * dd + 4) * 2.0 ** -24 * terms + 16 * 2.0 ** -23
