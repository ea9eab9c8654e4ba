"""Performance cases of the 4-bit distant cache: latents quantised as they are
written, a prefilled cache packed, both read back, and decode steps over it.

Four kinds of call:
  append  new tokens enter the cache: those that leave the window are projected
          (Eq. 1 of the paper) and quantised, the newest go to the ring; the rows
          written are read back
  pack    the latents of a prefilled cache are quantised, and read back
  read    the latents of a 4-bit cache are brought back to the cache's dtype
  decode  a decode step over ring and 4-bit latents (dense, or paged with a
          length per sequence)

A latent row is held in groups of 32 columns (the last may be shorter): per
group one byte E, the scale 2^(E - 127) being the smallest power of two s with
max |c| <= 7 s (within 2^-124 .. 2^125), per value four bits, sign and index
into 0, 1/2, 1, 3/2, 2, 3, 4, 6 of the nearest |c| / s (ties to the even index,
at most 6); two columns a byte, the even one in the low half, rows padded to
whole 32-bit words. What is held so is returned as the values it stands for.

With `own` false each is computed in elementary torch operations; exact()
restates the definitions in fp64, by the distance to every value of the format,
and lifts every distant token to full head dimension.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 64
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(kind, name=None, *, B, Hkv, T, d, dd, w, Hq=0, n=0, lo=0, dtype="bf16", untied=False,
          paged=False):
    """T: tokens held per sequence before the call; lo: of the shortest sequence
    of a ragged batch (0: all hold T); n: new tokens (append)."""
    c = dict(kind=kind, B=B, Hq=Hq or Hkv, Hkv=Hkv, T=T, n=n, d=d, dd=dd, w=w, lo=lo, dtype=dtype,
             untied=untied, paged=paged)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one conversation's next token, the window full: latency
        _case("append", "append_step", B=1, Hkv=8, T=331, n=1, d=64, dd=16, w=128),
        # continuous batching: a token for each of many sequences, in pages
        _case("append", "append_paged_d128", B=96, Hkv=8, T=1999, n=1, d=128, dd=32, w=1024, lo=300,
              paged=True),
        # prompts of a batch entering an empty cache at once
        _case("append", "append_prompt", B=8, Hkv=8, T=0, n=8191, d=64, dd=16, w=512),
        # a prefilled batch moves to 4 bits
        _case("pack", "pack_1b", B=16, Hkv=8, T=32768, d=64, dd=16, w=512),
        # the same in pages, ragged, a larger head
        _case("pack", "pack_ragged_d128", B=24, Hkv=8, T=16000, d=128, dd=32, w=1024, lo=1100,
              paged=True),
        # a finished turn of one conversation comes back for the next prompt: latency
        _case("read", "read_turn", B=1, Hkv=8, T=4501, d=64, dd=16, w=512),
        # a batch of long documents comes back
        _case("read", "read_docs_d128", B=4, Hkv=8, T=131072, d=128, dd=32, w=1024),
        # one short conversation, an odd length: latency
        _case("decode", "decode_short", B=1, Hq=8, Hkv=8, T=331, d=64, dd=16, w=128),
        # an fp32 reference run of a small model, a bottleneck of 20
        _case("decode", "decode_fp32", B=4, Hq=16, Hkv=4, T=4001, d=80, dd=20, w=256, dtype="f32"),
        # a full serving batch at 32K tokens of history
        _case("decode", "decode_1b", B=32, Hq=32, Hkv=8, T=32768, d=64, dd=16, w=512),
        # continuous batching, a larger head, W_up of its own: 1K to 16K tokens in pages
        _case("decode", "decode_ragged_d128", B=32, Hq=32, Hkv=8, T=16384, d=128, dd=32, w=1024,
              lo=1024, paged=True, untied=True),
        # one very long document, few KV heads
        _case("decode", "decode_long", B=1, Hq=32, Hkv=4, T=524287, d=128, dd=32, w=1024),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {"append": 1.6e8, "pack": 3.0e8, "read": 5.5e8, "decode": 1.8e8}
    while True:
        kind = rng.choice(["append", "pack", "read", "decode", "decode"])
        d = rng.choice([64, 64, 128])
        dd = rng.choice([16, 32])
        w = _log_int(rng, 32, 1024)
        Hkv = rng.choice([1, 2, 4, 8, 8])
        Hq = Hkv * rng.choice([1, 2, 4, 4, 7, 8])
        B = _log_int(rng, 1, 64)
        dtype, paged, untied, n = "bf16", rng.random() < 0.5, rng.random() < 0.3, 0
        if rng.random() < 0.2:  # the shapes that the matrix cores do not take
            dtype, d, dd = rng.choice(["f32", "f32", "bf16"]), rng.choice([64, 80, 128]), rng.choice([12, 16, 20, 33, 48])
            B = _log_int(rng, 1, 8)
        if kind == "append":
            T, n = rng.choice([0, _log_int(rng, 20, 4000)]), _log_int(rng, 1, 8192)
            if paged:
                T, n = _log_int(rng, 20, 4000), 1
        elif kind == "decode":
            T = _log_int(rng, 1, 262144) if rng.random() < 0.9 else _log_int(rng, 1, w)
        else:
            T = w + _log_int(rng, 1, 131072)
        lo = max(1, T // 16) if paged else 0
        c = _case(kind, B=B, Hq=Hq, Hkv=Hkv, T=T, n=n, d=d, dd=dd, w=w, lo=lo, dtype=dtype, untied=untied,
                  paged=paged)
        generic = dtype == "f32" or dd not in (16, 32) or d == 80
        wide = B * Hkv * dd * (T + n)
        if (work(c)["bytes"] <= most[kind] / (8 if generic and kind == "decode" else 1) and
                wide <= 1.4e8 and (kind != "decode" or B * Hq * T <= 34 * 10 ** 6) and
                (kind != "append" or (T + n > w and wide <= 2e7))):
            return c


# --- what a case holds --------------------------------------------------------

def _lens(c):
    """Tokens that the sequences hold before the call: spread evenly over the
    logarithm from lo to T (all T where lo is 0), long and short mixed."""
    B, T, lo = c["B"], c["T"], c["lo"]
    if not lo or B == 1:
        return [T] * B
    ls = [int(round(lo * (T / lo) ** (b / (B - 1)))) for b in range(B)]
    step = next(s for s in (13, 11, 7, 5, 3, 2, 1) if math.gcd(s, B) == 1)
    return [ls[(b * step + B - 1) % B] for b in range(B)]


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _blocks(c):
    return -(-(c["T"] + c["n"]) // PAGE)


def _store(c):
    """Shape of a latent array but for its columns: pages, or rows of a sequence."""
    if c["paged"]:
        return c["B"] * _blocks(c), c["Hkv"], PAGE
    return c["B"], c["Hkv"], c["T"] + c["n"]


def _row_bytes(dd):
    return 4 * (-(-dd // 8))


def _grid(x, step, most):
    """Values on a grid: every order of summing their products gives the same latent,
    so that none lies next to a rounding border by the order of a sum."""
    return (x / step).round().clamp(-most, most) * step


def _inputs(c, seed):
    """What a case holds. Keys, values and latents are unit normals (W_down keeps
    that scale), queries twice that, so that the softmax picks some tokens over
    others; a 4-bit cache holds quantised normals."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _dtype(c)
    B, Hq, Hkv, d, dd, w, n = (c[a] for a in ("B", "Hq", "Hkv", "d", "dd", "w", "n"))

    def normal(*shape, std=1.0):
        x = torch.randn(*shape, generator=g, device="cuda")
        return (x if std == 1.0 else x * std).to(dt)

    x = {}
    if c["kind"] == "append":
        for a, m in (("k_new", n), ("v_new", n), ("k_win", w), ("v_win", w)):
            x[a] = _grid(torch.randn(B, Hkv, m, d, generator=g, device="cuda"), 1 / 16, 127).to(dt)
        x["wd"] = _grid(torch.randn(Hkv, d, dd, generator=g, device="cuda") * d ** -0.5, 1 / 512, 255).to(dt)
    elif c["kind"] == "pack":
        x["k_lat"], x["v_lat"] = normal(*_store(c), dd), normal(*_store(c), dd)
    else:
        for a in "kv":
            x[a + "_codes"], x[a + "_exp"] = _quantise(normal(*_store(c), dd).float())
    if c["kind"] == "decode":
        x.update(q=normal(B, Hq, d, std=2.0), wd=normal(Hkv, d, dd, std=d ** -0.5),
                 wu=normal(Hkv, dd, d, std=dd ** -0.5) if c["untied"] else None,
                 k_win=normal(B, Hkv, w, d), v_win=normal(B, Hkv, w, d))
    if c["paged"]:
        pages = torch.randperm(B * _blocks(c), generator=torch.Generator().manual_seed(seed))
        x["table"] = pages.reshape(B, -1).to(torch.int32).contiguous().cuda()
    return x


def prepare(case, seed):
    c = case
    s = dict(_inputs(c, seed), case=c, back={})
    B, Hkv, d, dd, w = (c[a] for a in ("B", "Hkv", "d", "dd", "w"))
    s["lens"] = torch.tensor(_lens(c), dtype=torch.int32, device="cuda")
    s["first"] = (s["lens"] - w).clamp(min=0)
    if c["kind"] != "decode" and not own:
        s["back"] = {a: torch.zeros(*_store(c), dd, dtype=_dtype(c), device="cuda") for a in ("k_lat", "v_lat")}
    if own:
        import paper_2606_18587_amd as dar
        if c["paged"]:
            def make(cls):
                cache = cls(B, Hkv, d, dd, w, PAGE, _blocks(c), B * _blocks(c), _dtype(c))
                cache.block_table.copy_(s["table"])
                cache.lens.copy_(s["lens"])
                return cache
            plain, packed, names = dar.DarPagedCache, dar.DarPagedCacheQ4, ("k_pool", "v_pool")
        else:
            def make(cls):
                cache = cls(B, Hkv, d, dd, w, c["T"] + c["n"], _dtype(c))
                cache.struct.len = c["T"]
                return cache
            plain, packed, names = dar.DarCache, dar.DarCacheQ4, ("k_lat", "v_lat")
        s["cache"] = make(packed)
        for a in ("k_win", "v_win", "k_codes", "v_codes", "k_exp", "v_exp"):
            if a in s:  # (a dense cache holds its capacity rounded up to whole blocks)
                x = s.pop(a)
                getattr(s["cache"], a)[:, :, :x.shape[2]].copy_(x)
        if c["kind"] != "decode":
            s["to"] = make(plain)
            s["back"] = {"k_lat": getattr(s["to"], names[0]), "v_lat": getattr(s["to"], names[1])}
        if c["kind"] == "pack":
            s["from"] = make(plain)
            getattr(s["from"], names[0]).copy_(s.pop("k_lat"))
            getattr(s["from"], names[1]).copy_(s.pop("v_lat"))
    return s


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"append": _plain_append, "pack": _plain_pack, "read": _plain_read,
                "decode": _plain_decode}[c["kind"]](s, c)
    import paper_2606_18587_amd as dar
    cache = s["cache"]
    if c["kind"] == "decode":
        step = dar.dar_attn_decode_paged_q4 if c["paged"] else dar.dar_attn_decode_q4
        return {"o": step(cache, s["q"], s["wd"], s["wu"])}
    if c["kind"] == "append":
        if c["paged"]:
            cache.lens.copy_(s["lens"])  # where the sequences stand before the call
            dar.dar_cache_append_paged_q4(cache, s["k_new"][:, :, 0], s["v_new"][:, :, 0], s["wd"])
            dar.dar_cache_unpack_paged_q4(cache, s["to"], first=s["first"])
        else:
            cache.struct.len = c["T"]
            dar.dar_cache_append_q4(cache, s["k_new"], s["v_new"], s["wd"])
            dar.dar_cache_unpack_q4(cache, s["to"], first=max(c["T"] - c["w"], 0))
        return dict(s["back"], k_win=cache.k_win, v_win=cache.v_win,
                    lens=cache.lens if c["paged"] else cache.len)
    if c["kind"] == "pack":
        (dar.dar_cache_pack_paged_q4 if c["paged"] else dar.dar_cache_pack_q4)(s["from"], cache)
    (dar.dar_cache_unpack_paged_q4 if c["paged"] else dar.dar_cache_unpack_q4)(cache, s["to"])
    return dict(s["back"], lens=s["to"].lens if c["paged"] else s["to"].len)


# --- the operators in elementary operations -----------------------------------

def _groups(x):
    """x [..., dd] in groups of 32 columns, zeros behind the last: [..., groups, 32]."""
    dd = x.shape[-1]
    ng = -(-dd // 32)
    if dd < 32 * ng and dd > 32:
        x = torch.nn.functional.pad(x, (0, 32 * ng - dd))
    return x.reshape(*x.shape[:-1], ng, -1)


def _scale_byte(a):
    """E of groups whose largest absolute value is a (fp32)."""
    m, e = torch.frexp(a)
    E = e - 3 + 127 + (m > 0.875)
    return torch.where(a > 0, E, torch.zeros_like(E)).clamp(3, 252).to(torch.int32)


def _power(E):
    return (E.to(torch.int32) << 23).view(torch.float32)


def _indices(x):
    """Index 0..7 of the nearest level and sign bit of scaled values."""
    a = x.abs()
    i = torch.zeros(a.shape, dtype=torch.uint8, device=a.device)
    for k in range(7):
        mid = 0.5 * (LEVELS[k] + LEVELS[k + 1])
        i += (a >= mid) if k % 2 else (a > mid)  # a tie goes to the even index
    return i, (x < 0).to(torch.uint8) | ((x == 0) & torch.signbit(x)).to(torch.uint8)


def _quantise(x):
    """Bytes and scale bytes of rows x [..., dd] (fp32)."""
    dd = x.shape[-1]
    y = _groups(x)
    E = _scale_byte(y.abs().amax(-1))
    i, sign = _indices(y * _power(254 - E)[..., None])
    code = (i | (sign << 3)).reshape(*x.shape[:-1], -1)[..., :dd]
    code = torch.nn.functional.pad(code, (0, 2 * _row_bytes(dd) - dd))
    return (code[..., 0::2] | (code[..., 1::2] << 4)).contiguous(), E.to(torch.uint8)


def _values(codes, E, dd):
    """The rows (fp32) that bytes and scale bytes stand for."""
    i = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)[..., :dd].long()
    v = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=codes.device)[i]
    return v * _power(E).repeat_interleave(32, -1)[..., :dd]


def _held(x):
    """x as the cache gives it back."""
    y = _groups(x)
    s = _scale_byte(y.abs().amax(-1))
    z = y * _power(254 - s)[..., None]
    i, _ = _indices(z)
    v = torch.tensor(LEVELS, device=x.device)[i.long()]
    v = torch.where(torch.signbit(z), -v, v) * _power(s)[..., None]
    return v.reshape(*x.shape[:-1], -1)[..., :x.shape[-1]]


def _slot(s, pos):
    """Page and row of position pos [B, m] of every sequence."""
    return s["table"].long().gather(1, pos // PAGE), pos % PAGE


def _plain_append(s, c):
    B, Hkv, T, n, d, w = (c[a] for a in ("B", "Hkv", "T", "n", "d", "w"))
    lens = s["lens"].long()
    t = torch.arange(n, device="cuda")
    # the token that leaves the window as new token t enters it
    out = lens[:, None] + t - w
    old = (out < lens[:, None])[:, None, :, None]
    slot = (out % w)[:, None, :, None].expand(B, Hkv, n, d)
    came = (t - w).clamp(min=0)[None, None, :, None].expand(B, Hkv, n, d)
    up = s["wd"].double()
    for a in "kv":
        x = torch.where(old, s[a + "_win"].gather(2, slot), s[a + "_new"].gather(2, came))
        lat = torch.matmul(x.double(), up)  # 64 bits: which 4-bit value it takes hangs on its last bit
        v = _held(lat.to(s["wd"].dtype).float()).to(s["wd"].dtype)
        if c["paged"]:
            b = (out[:, 0] >= 0).nonzero()[:, 0]
            page, row = _slot(s, out.clamp(min=0))
            s["back"][a + "_lat"][page[b, 0], :, row[b, 0]] = v[b, :, 0]
        else:
            skip = max(w - T, 0)
            s["back"][a + "_lat"][:, :, T + skip - w:T + n - w] = v[:, :, skip:]
        last = min(n, w)
        to = ((lens[:, None] + t[n - last:]) % w)[:, None, :, None].expand(B, Hkv, last, d)
        s[a + "_win"].scatter_(2, to, s[a + "_new"][:, :, n - last:])
    return dict(s["back"], k_win=s["k_win"], v_win=s["v_win"],
                lens=(lens + n).to(torch.int32) if c["paged"] else T + n)


def _keep(s, c, a, v):
    """Rows v of the distant tokens into what is read back (the others stay)."""
    D = s["first"].long()
    if not c["paged"]:
        m = max(c["T"] - c["w"], 0)
        s["back"][a][:, :, :m] = v[:, :, :m]
        return
    at = torch.arange(_blocks(c) * PAGE, device="cuda")
    live = torch.zeros(c["B"] * _blocks(c), PAGE, dtype=torch.bool, device="cuda")
    live[s["table"].long()] = (at < D[:, None]).reshape(c["B"], -1, PAGE)
    s["back"][a].copy_(torch.where(live[:, None, :, None], v, s["back"][a]))


def _plain_pack(s, c):
    for a in ("k_lat", "v_lat"):
        _keep(s, c, a, _held(s[a].float()).to(s[a].dtype))
    return dict(s["back"], lens=s["lens"] if c["paged"] else c["T"])


def _plain_read(s, c):
    for a in "kv":
        v = _values(s[a + "_codes"], s[a + "_exp"], c["dd"]).to(_dtype(c))
        _keep(s, c, a + "_lat", v)
    return dict(s["back"], lens=s["lens"] if c["paged"] else c["T"])


def _plain_decode(s, c):
    B, Hq, Hkv, d, dd, w = (c[a] for a in ("B", "Hq", "Hkv", "d", "dd", "w"))
    G = Hq // Hkv
    near = s["lens"].long().clamp(max=w)
    far = s["lens"].long() - near
    wu = s["wd"].float().transpose(1, 2).contiguous() if s["wu"] is None else s["wu"].float()
    q = s["q"].float().reshape(B, Hkv, G, d)
    qt = q @ wu.transpose(1, 2).contiguous()
    k, v = (_values(s[a + "_codes"], s[a + "_exp"], dd) for a in "kv")
    if c["paged"]:
        k, v = (x[s["table"].long()].transpose(1, 2).reshape(B, Hkv, -1, dd) for x in (k, v))
    low = float("-inf")
    at = torch.arange(k.shape[2], device=q.device)
    sc = qt @ k.transpose(2, 3).contiguous()
    sc = sc.masked_fill(at >= far[:, None, None, None], low) / math.sqrt(d)
    # the window's tokens, oldest first
    i = torch.arange(w, device=q.device)
    slot = ((far[:, None] + i) % w)[:, None, :, None].expand(B, Hkv, w, d)
    kw, vw = (s[a].float().gather(2, slot) for a in ("k_win", "v_win"))
    sw = (q @ kw.transpose(2, 3).contiguous()).masked_fill(i >= near[:, None, None, None], low) / math.sqrt(d)
    m = torch.maximum(sc.amax(-1), sw.amax(-1))[..., None]
    pc, pw = torch.exp(sc - m), torch.exp(sw - m)
    o = pw @ vw + (pc @ v) @ wu
    o = o / (pc.sum(-1, keepdim=True) + pw.sum(-1, keepdim=True))
    return {"o": o.reshape(B, Hq, d).to(s["q"].dtype)}


# --- what a case cannot do without -------------------------------------------

def work(case):
    c = case
    B, Hq, Hkv, d, dd, w, n = (c[a] for a in ("B", "Hq", "Hkv", "d", "dd", "w", "n"))
    es = 2 if c["dtype"] == "bf16" else 4
    held = 2 * (_row_bytes(dd) + -(-dd // 32))  # a distant token of a KV head, key and value
    lat, row = 2 * dd * es, 2 * d * es
    nbytes, flops = 0.0, 0.0
    for L in _lens(c):
        far = max(L - w, 0)
        if c["kind"] == "append":
            leave = max(L + n - w, 0) - far
            ring = min(n, w)
            rows = n + min(leave, ring if L else 0)  # new tokens, and ring rows that leave
            # read; the ring's new rows; the 4-bit rows written and read again; their values
            nbytes += Hkv * (rows * row + ring * row + leave * (2 * held + lat))
            flops += Hkv * leave * 4 * d * dd
        elif c["kind"] == "pack":
            nbytes += Hkv * far * (2 * lat + 2 * held)
        elif c["kind"] == "read":
            nbytes += Hkv * far * (held + lat)
        else:
            near = min(L, w)
            nbytes += Hkv * (near * row + far * held)
            flops += Hq * (4 * d * near + 4 * dd * far)
    if c["kind"] in ("append", "decode"):
        nbytes += Hkv * d * dd * es * (2 if c["untied"] else 1)
    if c["kind"] == "decode":
        nbytes += 2 * B * Hq * d * es
    return {"bytes": nbytes, "flops": flops}


# --- the same in 64 bits ------------------------------------------------------

def _exact_held(x):
    """Rows x [..., dd] in fp64 as the format holds them: of every group the smallest
    power of two by trial, of every value the nearest level by its distance."""
    dd = x.shape[-1]
    levels = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    even = torch.tensor([0, 1e-12] * 4, dtype=torch.float64, device=x.device)  # ties: the even index first
    out = torch.empty_like(x)
    for g in range(0, dd, 32):
        y = x[..., g:g + 32]
        a = y.abs().amax(-1, keepdim=True)
        e = torch.floor(torch.log2(a.clamp(min=1e-300))) + 1
        for _ in range(5):
            e = torch.where(a <= 7 * torch.exp2(e - 1), e - 1, e)
        s = torch.exp2(e.clamp(-124, 125))
        near = ((y.abs() / s)[..., None] - levels).abs().add_(even).argmin(-1)
        out[..., g:g + 32] = torch.copysign(levels[near], y) * s
    return out


def _exact_values(codes, E, dd):
    out = torch.zeros(*codes.shape[:-1], dd, dtype=torch.float64, device=codes.device)
    for j in range(dd):
        nib = (codes[..., j // 2].int() >> (4 * (j % 2))) & 15
        e, m = (nib >> 1) & 3, nib & 1
        v = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * torch.exp2(e.double() - 1))
        out[..., j] = torch.where(nib >= 8, -v, v) * torch.exp2(E[..., j // 32].double() - 127)
    return out


def _exact_at(c, x, b, e):
    """Index of tokens e of sequence b in a latent array."""
    return (x["table"][b, e // PAGE].long(), slice(None), e % PAGE) if c["paged"] else (b, slice(None), e)


def exact(case, seed):
    c = case
    x = _inputs(c, seed)
    if c["kind"] == "decode":
        return _exact_decode(c, x)
    B, Hkv, n, w, dd = (c[a] for a in ("B", "Hkv", "n", "w", "dd"))
    out = {a: torch.zeros(*_store(c), dd, dtype=torch.float64, device="cuda") for a in ("k_lat", "v_lat")}
    for a in "kv":
        if c["kind"] == "append":
            ring = x[a + "_win"].double()
            for b, L in enumerate(_lens(c)):
                # the sequence's tokens from the window's first one on
                first = max(L - w, 0)
                seen = ring[b, :, torch.arange(first, L, device="cuda") % w]
                seen = torch.cat([seen, x[a + "_new"][b].double()], 1)
                m = max(L + n - w, 0) - first
                lat = torch.bmm(seen[:, :m], x["wd"].double()).to(_dtype(c)).double()
                at = _exact_at(c, x, b, torch.arange(first, first + m, device="cuda"))
                rows = _exact_held(lat)
                out[a + "_lat"][at] = rows.transpose(0, 1) if c["paged"] else rows
                p = torch.arange(L + n - min(n, w), L + n, device="cuda")
                ring[b, :, p % w] = seen[:, p - first]
            out[a + "_win"] = ring
            continue
        y = (_exact_held(x[a + "_lat"].double()) if c["kind"] == "pack" else
             _exact_values(x[a + "_codes"], x[a + "_exp"], dd))
        for b, L in enumerate(_lens(c)):
            at = _exact_at(c, x, b, torch.arange(max(L - w, 0), device="cuda"))
            out[a + "_lat"][at] = y[at]
    L = [v + n for v in _lens(c)]
    out["lens"] = torch.tensor(L, dtype=torch.int32) if c["paged"] else L[0]
    return out


def _exact_decode(c, x):
    B, Hq, Hkv, d, dd, w = (c[a] for a in ("B", "Hq", "Hkv", "d", "dd", "w"))
    G = Hq // Hkv
    up = x["wd"].double().transpose(1, 2).contiguous() if x["wu"] is None else x["wu"].double()
    o = torch.zeros(B, Hq, d, dtype=torch.float64, device="cuda")
    for b, L in enumerate(_lens(c)):
        far = max(L - w, 0)
        slots = torch.arange(far, L, device="cuda") % w
        at = _exact_at(c, x, b, torch.arange(far, device="cuda"))
        kv = []
        for a in "kv":
            codes, E = x[a + "_codes"][at], x[a + "_exp"][at]
            if c["paged"]:
                codes, E = codes.transpose(0, 1).contiguous(), E.transpose(0, 1).contiguous()
            lift = torch.bmm(_exact_values(codes, E, dd), up)
            kv.append(torch.cat([lift, x[a + "_win"][b][:, slots].double()], 1))
        for g in range(Hkv):
            s = x["q"][b, g * G:(g + 1) * G].double() @ kv[0][g].t().contiguous() / d ** 0.5
            o[b, g * G:(g + 1) * G] = torch.softmax(s, dim=1) @ kv[1][g]
    return {"o": o}
