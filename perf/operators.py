"""Performance cases of the serving operators: decode steps that score the cached
tokens by the attention weight they receive, eviction of the least attended
ones, and decode steps of a batch whose sequences share a long prefix.

Three kinds of call:
  scored  a decode step that also adds every cached token's attention weight,
          summed over the query heads of its KV head, to a score (dense cache,
          or paged with a length per sequence, with or without a shared prefix)
  evict   the distant tokens with the lowest scores leave the cache: the kept
          ones past its new end move into the slots that become free
  prefix  a decode step over a paged cache whose sequences share their first P
          tokens, kept once

With `own` false each is computed in elementary torch operations in fp32;
exact() restates the definitions in fp64, lifting every distant token to full
head dimension (Eq. 2-4 of the paper) instead of absorbing W_up.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 64


def _case(kind, name=None, *, B, Hq, Hkv, T, d, dd, w, dtype="bf16", untied=False, paged=False,
          lo=0, P=0, keep=0, fixed=0):
    """T: tokens cached per sequence (after the shared prefix, if there is one);
    lo: of the shortest sequence of a ragged batch (0: all hold T); P: shared
    prefix tokens; keep, fixed: distant tokens an eviction keeps at least, and
    how many of the first are never evicted."""
    c = dict(kind=kind, B=B, Hq=Hq, Hkv=Hkv, T=T, d=d, dd=dd, w=w, dtype=dtype, untied=untied,
             paged=paged, lo=lo, P=P, keep=keep, fixed=fixed)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one short conversation, an odd length: latency
        _case("scored", "scored_short", B=1, Hq=8, Hkv=8, T=331, d=64, dd=16, w=128),
        # an fp32 reference run of a small model
        _case("scored", "scored_fp32", B=4, Hq=16, Hkv=4, T=4001, d=64, dd=16, w=256, dtype="f32"),
        # a full serving batch at 32K tokens of history
        _case("scored", "scored_1b", B=32, Hq=32, Hkv=8, T=32768, d=64, dd=16, w=512),
        # continuous batching, a larger head, W_up of its own: 1K to 16K tokens in pages
        _case("scored", "scored_ragged_d128", B=32, Hq=32, Hkv=8, T=16384, d=128, dd=32, w=1024,
              paged=True, lo=1024, untied=True),
        # many sequences after a shared prompt whose own tokens are scored
        _case("scored", "scored_prefix", B=48, Hq=32, Hkv=8, T=4500, d=64, dd=16, w=512, paged=True,
              lo=700, P=16384),
        # a few sequences just over a small budget: latency
        _case("evict", "evict_small", B=2, Hq=8, Hkv=8, T=2451, d=64, dd=16, w=128, keep=2048,
              fixed=4),
        # a full serving batch kept at 32K tokens: one window's worth leaves
        _case("evict", "evict_1b", B=32, Hq=32, Hkv=8, T=33999, d=64, dd=16, w=512, keep=32768,
              fixed=4),
        # long documents cut to half their length after the prompt
        _case("evict", "evict_halve_d128", B=8, Hq=32, Hkv=8, T=131072, d=128, dd=32, w=1024,
              keep=65536),
        # continuous batching: sequences of 2K to 32K tokens in pages, brought under one budget
        _case("evict", "evict_ragged", B=32, Hq=32, Hkv=8, T=32768, d=64, dd=16, w=512, paged=True,
              lo=2048, keep=8192, fixed=64),
        # a few requests on a short system prompt, some shorter than the window: latency
        _case("prefix", "prefix_small", B=4, Hq=8, Hkv=8, T=203, d=64, dd=16, w=128, paged=True,
              lo=17, P=512),
        # a serving batch on one long document
        _case("prefix", "prefix_32k", B=64, Hq=32, Hkv=8, T=2500, d=64, dd=16, w=512, paged=True,
              lo=600, P=32768),
        # a larger head, W_up of its own, conversations longer than their prompt
        _case("prefix", "prefix_d128", B=24, Hq=32, Hkv=4, T=12000, d=128, dd=32, w=1024, paged=True,
              lo=1100, P=8192, untied=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {"scored": 6.0e8, "evict": 5.0e8, "prefix": 1.0e8}
    while True:
        kind = rng.choice(["scored", "scored", "evict", "prefix"])
        d = rng.choice([64, 64, 128])
        dd = rng.choice([16, 32])
        w = _log_int(rng, 32, 1024)
        Hkv = rng.choice([2, 4, 8, 8])
        Hq = Hkv * rng.choice([1, 2, 4, 4, 8])
        untied = rng.random() < 0.3
        if kind == "scored":
            paged = rng.random() < 0.5
            T = _log_int(rng, 200, 32768)
            if rng.random() < 0.2:  # the shapes that the matrix-core decode does not take
                c = _case(kind, B=_log_int(rng, 1, 8), Hq=Hq, Hkv=Hkv, T=_log_int(rng, 200, 8192),
                          d=rng.choice([64, 80, 128]), dd=rng.choice([16, 20]), w=w, dtype="f32",
                          untied=untied)
            else:
                P = PAGE * _log_int(rng, 4, 256) if paged and rng.random() < 0.5 else 0
                c = _case(kind, B=_log_int(rng, 1, 64), Hq=Hq, Hkv=Hkv, T=T, d=d, dd=dd, w=w,
                          untied=untied, paged=paged, lo=max(1, T // 16) if paged else 0, P=P)
        elif kind == "evict":
            paged = rng.random() < 0.5
            T = _log_int(rng, 1500, 131072)
            keep = int(T * rng.uniform(0.3, 0.95))
            c = _case(kind, B=_log_int(rng, 1, 32), Hq=Hq, Hkv=Hkv, T=T, d=d, dd=dd, w=w,
                      paged=paged, lo=max(1, T // 16) if paged else 0, keep=keep,
                      fixed=rng.choice([0, 4, 64, keep // 2]))
        else:
            T = _log_int(rng, 50, 8192)
            c = _case(kind, B=_log_int(rng, 2, 96), Hq=Hq, Hkv=Hkv, T=T, d=d, dd=dd, w=w,
                      untied=untied, paged=True, lo=max(1, T // 16), P=PAGE * _log_int(rng, 4, 512))
        heads = c["B"] * (c["Hkv"] if kind == "evict" else c["Hq"])
        if (work(c)["bytes"] <= most[kind] and heads * c["P"] <= 64 * 32 * 32768 and
                heads * c["T"] <= (12 if kind == "evict" else 40) * 10 ** 6):
            return c


# --- what a case holds --------------------------------------------------------

def _lens(c):
    """Tokens of a batch's sequences, the shared prefix among them: spread evenly
    over the logarithm from lo to T (all T where lo is 0), in an order that
    mixes long and short."""
    B, T, lo = c["B"], c["T"], c["lo"]
    if not lo or B == 1:
        return [c["P"] + T] * B
    ls = [int(round(lo * (T / lo) ** (b / (B - 1)))) for b in range(B)]
    step = next(s for s in (13, 11, 7, 5, 3, 2, 1) if math.gcd(s, B) == 1)
    return [c["P"] + ls[(b * step + B - 1) % B] for b in range(B)]


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _blocks(c):
    """Pages of the shared prefix, pages of a sequence's own tokens, slots of a
    sequence."""
    shared, rest = c["P"] // PAGE, -(-c["T"] // PAGE)
    return shared, rest, (shared + rest) * PAGE


def _slots(c):
    return _blocks(c)[2] if c["paged"] else c["T"]


def _inputs(c, seed):
    """Query, weights, cache and scores of a case. Keys, values and latents are
    unit normals (W_down keeps that scale); queries twice that, so that the
    softmax picks some tokens over others; scores are sums of many steps'
    weights, a few tokens far above the rest, some never attended."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _dtype(c)
    B, Hq, Hkv, d, dd, w = (c[x] for x in ("B", "Hq", "Hkv", "d", "dd", "w"))

    def normal(*shape, std=1.0):
        x = torch.randn(*shape, generator=g, device="cuda", dtype=dt)
        return x if std == 1.0 else x * std

    shared, rest, slots = _blocks(c)
    rows = (shared + rest * B, Hkv, PAGE, dd) if c["paged"] else (B, Hkv, c["T"], dd)
    x = {"q": normal(B, Hq, d, std=2.0), "wd": normal(Hkv, d, dd, std=d ** -0.5),
         "wu": normal(Hkv, dd, d, std=dd ** -0.5) if c["untied"] else None,
         "k_win": normal(B, Hkv, w, d), "v_win": normal(B, Hkv, w, d),
         "k_lat": normal(*rows), "v_lat": normal(*rows)}
    if c["kind"] != "prefix":
        z = torch.randn(B, Hkv, _slots(c), generator=g, device="cuda")
        z = torch.exp(1.5 * z) * (z > -2.2) * (256.0 / c["T"])
        z[torch.arange(_slots(c), device="cuda") >= torch.tensor(_lens(c), device="cuda")[:, None, None]
          .expand_as(z)] = 0.0
        x["scores"] = z
    if c["paged"]:
        pages = torch.randperm(rows[0], generator=torch.Generator().manual_seed(seed))
        table = torch.cat([pages[:shared].expand(B, shared), pages[shared:].reshape(B, rest)], 1)
        x["table"] = table.to(torch.int32).contiguous().cuda()
    return x


def prepare(case, seed):
    c = case
    s = dict(_inputs(c, seed), case=c)
    s["lens"] = torch.tensor(_lens(c), dtype=torch.int32, device="cuda")
    s["end"] = max(_lens(c))
    if "scores" in s:
        s["scores_out"] = torch.zeros_like(s["scores"])
    if own:
        import paper_2606_18587_amd as dar
        if c["paged"]:
            cache = dar.DarPagedCache(c["B"], c["Hkv"], c["d"], c["dd"], c["w"], PAGE,
                                      s["table"].shape[1], s["k_lat"].shape[0], _dtype(c))
            cache.block_table.copy_(s["table"])
            cache.lens.copy_(s["lens"])
            names = ("k_pool", "v_pool")
        else:
            cache = dar.DarCache(c["B"], c["Hkv"], c["d"], c["dd"], c["w"], c["T"], _dtype(c))
            cache.struct.len = c["T"]
            names = ("k_lat", "v_lat")
        for to, a in (("k_win", "k_win"), ("v_win", "v_win"), (names[0], "k_lat"), (names[1], "v_lat")):
            getattr(cache, to).copy_(s.pop(a))
        s["cache"] = cache
    return s


def run(state):
    s, c = state, state["case"]
    if not own:
        return _plain_evict(s, c) if c["kind"] == "evict" else _plain_decode(s, c)
    import paper_2606_18587_amd as dar
    cache = s["cache"]
    shared = s["table"][0, :c["P"] // PAGE] if c["P"] else None
    if c["kind"] == "prefix":
        return {"o": dar.dar_attn_decode_paged_prefix(cache, s["q"], s["wd"], shared, s["wu"])}
    if c["kind"] == "scored":
        if c["paged"]:
            o = dar.dar_attn_decode_paged_scored(cache, s["q"], s["wd"], s["scores"], s["wu"],
                                                 prefix_blocks=shared, scores_out=s["scores_out"])
        else:
            o = dar.dar_attn_decode_scored(cache, s["q"], s["wd"], s["scores"], s["wu"],
                                           scores_out=s["scores_out"])
        return {"o": o, "scores": s["scores_out"]}
    if c["paged"]:
        cache.lens.copy_(s["lens"])  # where the appends since the last eviction have brought them
        dar.dar_cache_evict_paged(cache, s["scores"], c["keep"], n_fixed=c["fixed"],
                                  scores_out=s["scores_out"])
        return {"k_lat": cache.k_pool, "v_lat": cache.v_pool, "scores": s["scores_out"],
                "lens": cache.lens}
    cache.struct.len = c["T"]  # where the appends since the last eviction have brought it
    dar.dar_cache_evict(cache, s["scores"], c["keep"], n_fixed=c["fixed"],
                        scores_out=s["scores_out"])
    return {"k_lat": cache.k_lat, "v_lat": cache.v_lat, "scores": s["scores_out"], "lens": cache.len}


# --- the operators in elementary operations -----------------------------------

def _rows(pool, table):
    """Rows of the pages that `table` [B, n] names, in order: [B, Hkv, n PAGE, dd]."""
    x = pool[table.long()]
    return x.transpose(1, 2).reshape(x.shape[0], x.shape[2], -1, x.shape[4])


def _plain_decode(s, c):
    B, Hq, Hkv, d, w, P = (c[x] for x in ("B", "Hq", "Hkv", "d", "w", "P"))
    G = Hq // Hkv
    near = s["lens"].long().clamp(max=w)
    far = s["lens"].long() - near          # distant tokens
    wu = s["wd"].float().transpose(1, 2).contiguous() if s["wu"] is None else s["wu"].float()
    q = s["q"].float().reshape(B, Hkv, G, d)
    qt = q @ wu.transpose(1, 2).contiguous()
    if c["paged"]:
        k, v = (_rows(s[a], s["table"][:, P // PAGE:]).float() for a in ("k_lat", "v_lat"))
    else:
        k, v = s["k_lat"].float(), s["v_lat"].float()
    n = k.shape[2]
    at = P + torch.arange(n, device=q.device)
    low = float("-inf")
    sc = qt @ k.transpose(2, 3).contiguous()
    parts = [sc.masked_fill(at >= far[:, None, None, None], low)]
    # the window's tokens, oldest first
    i = torch.arange(w, device=q.device)
    slot = ((far[:, None] + i) % w)[:, None, :, None].expand(B, Hkv, w, d)
    kw, vw = (s[a].float().gather(2, slot) for a in ("k_win", "v_win"))
    sc = q @ kw.transpose(2, 3).contiguous()
    parts.append(sc.masked_fill(i >= near[:, None, None, None], low))
    if P:
        pre = s["table"][:1, :P // PAGE]
        kp, vp = (_rows(s[a], pre)[0].float() for a in ("k_lat", "v_lat"))
        rows = qt.transpose(0, 1).reshape(Hkv, B * G, -1)
        sc = (rows @ kp.transpose(1, 2).contiguous()).reshape(Hkv, B, G, P).transpose(0, 1)
        parts.append(sc.masked_fill(torch.arange(P, device=q.device) >= far[:, None, None, None], low))
    parts = [x / math.sqrt(d) for x in parts]
    m = torch.stack([x.amax(-1) for x in parts]).amax(0)[..., None]
    parts = [torch.exp(x - m) for x in parts]
    total = sum(x.sum(-1) for x in parts)[..., None]
    lat = parts[0] @ v
    if P:
        p = parts[2].transpose(0, 1).reshape(Hkv, B * G, P)
        lat = lat + (p @ vp).reshape(Hkv, B, G, -1).transpose(0, 1)
    o = ((parts[1] @ vw + lat @ wu) / total).reshape(B, Hq, d).to(s["q"].dtype)
    if c["kind"] == "prefix":
        return {"o": o}
    out = s["scores"].clone()
    out[:, :, P:P + n] += (parts[0] / total).sum(2)
    pos = (far[:, None] + i).clamp(max=out.shape[2] - 1)
    mine = (pos >= P) & (i < near[:, None])
    out.scatter_add_(2, pos[:, None].expand(B, Hkv, w), (parts[1] / total).sum(2) * mine[:, None])
    if P:
        out[:, :, :P] = 0.0  # the prefix has no scores
    return {"o": o, "scores": out}


def _plain_evict(s, c):
    B, Hkv, w, keep, fixed = (c[x] for x in ("B", "Hkv", "w", "keep", "fixed"))
    z = s["scores"]
    n = z.shape[2]
    at = torch.arange(n, device=z.device)
    lens = s["lens"].long()[:, None, None]
    D = (lens - w).clamp(min=0)
    E = (D - keep).clamp(min=0) // w * w
    left = D - E
    # rank of every distant token: the fixed ones first, then by score, then by slot
    key = torch.where(at < D, z, -1.0).masked_fill(at < fixed, float("inf"))
    order = torch.argsort(key, dim=2, descending=True, stable=True)
    rank = torch.empty_like(order).scatter_(2, order, at.expand_as(order).contiguous())
    kept = (rank < left) & (at < D)
    hole = ~kept & (at < left)
    tail = kept & (at >= left)
    tails = torch.argsort((~tail).to(torch.int8), dim=2, stable=True)  # their slots, ascending
    nth = (torch.cumsum(hole, 2) - 1).clamp(min=0)
    src = torch.where(hole, tails.gather(2, nth), at)
    new = torch.where(at < left, z.gather(2, src), 0.0)
    near = (at >= left) & (at < lens - E)
    new = torch.where(near, z.gather(2, (at + E).clamp(max=n - 1).expand_as(src)), new)
    out = {"scores": new}
    if c["paged"]:
        page, row = s["table"].long()[:, at // PAGE][:, None, :], at % PAGE
        g = torch.arange(Hkv, device=z.device)[None, :, None]
        for a in ("k_lat", "v_lat"):
            x = _rows(s[a], s["table"])
            x = x.gather(2, src[..., None].expand_as(x))
            s[a][page, g, row] = x
            out[a] = s[a]
        out["lens"] = (lens - E)[:, 0, 0].to(torch.int32)
        return out
    for a in ("k_lat", "v_lat"):
        out[a] = s[a].gather(2, src[..., None].expand_as(s[a]))
    D = max(c["T"] - w, 0)
    out["lens"] = c["T"] - max(D - keep, 0) // w * w
    return out


# --- what a case cannot do without -------------------------------------------

def work(case):
    c = case
    B, Hq, Hkv, d, dd, w, P = (c[x] for x in ("B", "Hq", "Hkv", "d", "dd", "w", "P"))
    es = 2 if c["dtype"] == "bf16" else 4
    nbytes = flops = 0.0
    if c["kind"] == "evict":
        for n in _lens(c):
            D = max(n - w, 0)
            E = max(D - c["keep"], 0) // w * w
            # scores that do not go by the slot: this many kept tokens change places
            moved = E * max(D - E - c["fixed"], 0) / max(D - c["fixed"], 1)
            # scores read and written, rows read and written
            nbytes += Hkv * (4 * n + 4 * (n - E) + moved * 4 * dd * es)
        return {"bytes": nbytes, "flops": 0}
    for n in _lens(c):
        near = min(n, w)
        alone = max(n - near - P, 0)                 # distant tokens of this sequence's own
        nbytes += Hkv * 2 * es * (near * d + alone * dd)
        flops += Hq * (4 * d * near + 4 * dd * (n - near))
        if c["kind"] == "scored":
            nbytes += Hkv * 8 * (n - P)
    nbytes += Hkv * 2 * es * P * dd + 2 * B * Hq * d * es + Hkv * d * dd * es * (2 if c["untied"] else 1)
    return {"bytes": nbytes, "flops": flops}


# --- the same in 64 bits ------------------------------------------------------

def exact(case, seed):
    c, x = case, _inputs(case, seed)
    return _exact_evict(c, x) if c["kind"] == "evict" else _exact_decode(c, x)


def _own_rows(c, x, name, b, n):
    """Latent rows [Hkv, n, dd] of sequence b's first n tokens."""
    if not c["paged"]:
        return x[name][b, :, :n].double()
    e = torch.arange(n, device="cuda")
    return x[name][x["table"][b, e // PAGE].long(), :, e % PAGE].double().transpose(0, 1).contiguous()


def _exact_decode(c, x):
    B, Hq, Hkv, d, w = (c[a] for a in ("B", "Hq", "Hkv", "d", "w"))
    G = Hq // Hkv
    up = x["wd"].double().transpose(1, 2).contiguous() if x["wu"] is None else x["wu"].double()
    o = torch.zeros(B, Hq, d, dtype=torch.float64, device="cuda")
    scores = x["scores"].double() if "scores" in x else None
    for b, n in enumerate(_lens(c)):
        far = max(n - w, 0)
        slots = torch.arange(far, n, device="cuda") % w
        k, v = (torch.cat([torch.bmm(_own_rows(c, x, lat, b, far), up), x[win][b, :, slots].double()], 1)
                for lat, win in (("k_lat", "k_win"), ("v_lat", "v_win")))
        for g in range(Hkv):
            s = x["q"][b, g * G:(g + 1) * G].double() @ k[g].t().contiguous() / d ** 0.5
            p = torch.softmax(s, dim=1)
            o[b, g * G:(g + 1) * G] = p @ v[g]
            if scores is not None:
                scores[b, g, c["P"]:n] += p[:, c["P"]:].sum(0)
    if scores is None:
        return {"o": o}
    scores[:, :, :c["P"]] = 0.0
    return {"o": o, "scores": scores}


def _exact_evict(c, x):
    B, Hkv, w, fixed = (c[a] for a in ("B", "Hkv", "w", "fixed"))
    z = x["scores"].cpu().numpy()
    new = np.zeros_like(z)
    slots = z.shape[2]
    src = np.tile(np.arange(slots), (B, Hkv, 1))
    lens = []
    for b, n in enumerate(_lens(c)):
        D = max(n - w, 0)
        E = (max(D - c["keep"], 0) // w) * w
        lens.append(n - E)
        for g in range(Hkv):
            first = min(fixed, D)
            best = first + np.lexsort((np.arange(D - first), -z[b, g, first:D]))[:D - E - first]
            stay = np.zeros(D, bool)
            stay[:first] = True
            stay[best] = True
            free = np.flatnonzero(~stay[:D - E])
            src[b, g, free] = D - E + np.flatnonzero(stay[D - E:])
            new[b, g, :D - E] = z[b, g, src[b, g, :D - E]]
            new[b, g, D - E:n - E] = z[b, g, D:n]
    out = {"scores": torch.from_numpy(new).double(),
           "lens": torch.tensor(lens, dtype=torch.int32) if c["paged"] else lens[0]}
    at = torch.from_numpy(src).cuda()
    for a in ("k_lat", "v_lat"):
        if c["paged"]:
            y = x[a].double()
            for b in range(B):
                rows = _own_rows(c, x, a, b, slots)
                rows = rows.gather(1, at[b][..., None].expand_as(rows))
                e = torch.arange(slots, device="cuda")
                y[x["table"][b, e // PAGE].long(), :, e % PAGE] = rows.transpose(0, 1)
            out[a] = y
        else:
            out[a] = x[a].gather(2, at[..., None].expand_as(x[a])).double()
    return out
