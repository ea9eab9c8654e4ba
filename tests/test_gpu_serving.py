"""The serving operators together, as a server uses them: a prompt prefilled
once into pages that every sequence of a batch shares, then steps of append,
scored decode after the shared prefix and, when a budget is passed, eviction
behind it. Every step's output is compared with the definition over the tokens
that should be left (fp64, from the tokens themselves, not from the cache).
Captured graphs, other streams and several users of one GPU follow."""
import numpy as np
import pytest
import torch

from tests.dev import tol
from tests.serving_ref import f64
from tests.test_gpu_evict import counts, reference

pytestmark = pytest.mark.gpu

dar = pytest.importorskip("paper_2606_18587_amd")

BF = torch.bfloat16


def definition(q, k, v, wd, up, near):
    """q [G,d] over tokens k, v [n,d], the last `near` of them in the window."""
    n, d = k.shape
    far = np.arange(n) < n - near
    kk = np.where(far[:, None], k @ wd @ up, k)
    vv = np.where(far[:, None], v @ wd @ up, v)
    s = q @ kk.T / np.sqrt(d)
    p = np.exp(s - s.max(1, keepdims=True))
    return p / p.sum(1, keepdims=True) @ vv


@pytest.mark.parametrize("d,dd,G,w,ps", [(64, 16, 4, 32, 32), (128, 32, 2, 48, 64)])
def test_server_loop(d, dd, G, w, ps):
    B, Hkv, n0, steps, budget = 5, 2, 300, 150, 40
    Hq = Hkv * G
    g = torch.Generator().manual_seed(d)
    wd = (torch.randn(Hkv, d, dd, generator=g) * d ** -0.5).to(BF)
    prompt = [torch.randn(1, Hkv, n0, d, generator=g).to(BF) for _ in range(2)]
    new = [torch.randn(steps, B, Hkv, d, generator=g).to(BF) for _ in range(2)]
    qs = (torch.randn(steps, B, Hq, d, generator=g) * 2).to(BF)

    # the prompt goes in once, into sequence 0 of a one-sequence view of the pool
    shared = (n0 - w) // ps              # whole pages of tokens that are distant already
    P = shared * ps
    own = -(-(n0 + steps - P) // ps) + 1
    c = dar.DarPagedCache(B, Hkv, d, dd, w, ps, shared + own, shared + B * own, BF)
    bt = torch.cat([torch.arange(shared).expand(B, shared),
                    shared + torch.arange(B * own).reshape(B, own)], 1).to(torch.int32)
    c.block_table.copy_(bt)
    one = dar.DarPagedCache(1, Hkv, d, dd, w, ps, shared + own, shared + B * own, BF)
    one.k_pool, one.v_pool = c.k_pool, c.v_pool
    one.block_table.copy_(bt[:1])
    dar.dar_attn_prefill_chunk_paged(one, torch.zeros(1, Hq, n0, d, dtype=BF, device="cuda"),
                                     prompt[0].cuda(), prompt[1].cuda(), wd.cuda())
    # the others take its ring, its length and a copy of the page that is not full
    for t, x in ((c.k_win, one.k_win), (c.v_win, one.v_win)):
        t.copy_(x.expand_as(t))
    c.lens.fill_(n0)
    for pool in (c.k_pool, c.v_pool):
        pool[bt[1:, shared].long().cuda()] = pool[int(bt[0, shared])].clone()
    blocks = c.block_table[0, :shared]

    wd64 = f64(wd)
    ids = np.tile(np.arange(n0), (B, Hkv, 1))      # token in every slot, prompt first
    k = np.stack([np.concatenate([f64(prompt[0])[0], f64(new[0])[:, b].transpose(1, 0, 2)], 1) for b in range(B)])
    v = np.stack([np.concatenate([f64(prompt[1])[0], f64(new[1])[:, b].transpose(1, 0, 2)], 1) for b in range(B)])
    scores = torch.zeros(B, Hkv, c.cap, device="cuda")
    n, evictions = n0, 0
    for t in range(steps):
        dar.dar_cache_append_paged(c, new[0][t].cuda(), new[1][t].cuda(), wd.cuda(), Hq=Hq)
        ids = np.concatenate([ids, np.full((B, Hkv, 1), n0 + t)], 2)
        n += 1
        q = qs[t].cuda()
        o = f64(dar.dar_attn_decode_paged_scored(c, q, wd.cuda(), scores, prefix_blocks=blocks))
        if t % 7 == 0 or t == steps - 1:
            for b in range(B):
                for h in range(Hkv):
                    hs = slice(h * G, (h + 1) * G)
                    want = definition(f64(q)[b, hs], k[b, h, ids[b, h]], v[b, h, ids[b, h]], wd64[h],
                                      wd64[h].T, w)
                    assert np.abs(o[b, hs] - want).max() <= tol("bf16"), (t, b, h)
        E = counts(n, w, P + budget)[1]
        if E:
            z = scores.cpu().numpy()
            dar.dar_cache_evict_paged(c, scores, P + budget, n_fixed=P)
            kept = np.empty((B, Hkv, n - E), np.int64)
            for b in range(B):
                for h in range(Hkv):
                    src, after, _ = reference(z[b, h], n, w, P + budget, P)
                    row = ids[b, h, np.concatenate([src[:n - E - w], np.arange(n - w, n)])]
                    assert len(set(row)) == n - E and set(range(P)) <= set(row)
                    kept[b, h] = row
                    assert np.array_equal(scores[b, h].cpu().numpy()[:n], after[:n])
            ids, n, evictions = kept, n - E, evictions + 1
            assert c.lens.cpu().tolist() == [n] * B
    assert evictions >= 2
    assert (scores[:, :, n:] == 0).all() and (scores[:, :, :P] == 0).all()


def test_dense_loop():
    """Append, scored decode and eviction over a dense cache; the plain decode and
    the chunked prefill then read the evicted cache like any other."""
    B, Hq, Hkv, d, dd, w, steps, budget = 2, 4, 2, 64, 16, 16, 90, 30
    g = torch.Generator().manual_seed(8)
    wd = (torch.randn(Hkv, d, dd, generator=g) * d ** -0.5).to(BF)
    k, v = (torch.randn(B, Hkv, steps + 20, d, generator=g).to(BF) for _ in range(2))
    c = dar.DarCache(B, Hkv, d, dd, w, 128, BF)
    scores = torch.zeros(B, Hkv, 128, device="cuda")
    ids = np.zeros((B, Hkv, 0), np.int64)
    gone = 0

    def compare(o, q):
        for b in range(B):
            for h in range(Hkv):
                hs = slice(2 * h, 2 * h + 2)
                want = definition(f64(q)[b, hs], f64(k)[b, h, ids[b, h]], f64(v)[b, h, ids[b, h]],
                                  f64(wd)[h], f64(wd)[h].T, min(w, ids.shape[2]))
                assert np.abs(f64(o)[b, hs] - want).max() <= tol("bf16")

    for t in range(steps):
        dar.dar_cache_append(c, k[:, :, t:t + 1].contiguous().cuda(), v[:, :, t:t + 1].contiguous().cuda(),
                             wd.cuda(), Hq=Hq)
        ids = np.concatenate([ids, np.full((B, Hkv, 1), t)], 2)
        q = (torch.randn(B, Hq, d, generator=g) * 2).to(BF).cuda()
        compare(dar.dar_attn_decode_scored(c, q, wd.cuda(), scores), q)
        compare(dar.dar_attn_decode(c, q, wd.cuda()), q)
        n, z = c.len, scores.cpu().numpy()
        E = dar.dar_cache_evict(c, scores, budget, n_fixed=2)
        gone += E
        if E:
            ids = np.stack([np.stack([ids[b, h][np.concatenate([
                reference(z[b, h], n, w, budget, 2)[0][:n - E - w], np.arange(n - w, n)])]
                for h in range(Hkv)]) for b in range(B)])
    assert gone >= 2 * w and c.len == steps - gone
    # a chunk of new tokens onto the evicted cache
    q = (torch.randn(B, Hq, 20, d, generator=g) * 2).to(BF).cuda()
    o = dar.dar_attn_prefill_chunk(c, q, k[:, :, steps:].contiguous().cuda(), v[:, :, steps:].contiguous().cuda(),
                                   wd.cuda())
    for i in range(20):
        ids = np.concatenate([ids, np.full((B, Hkv, 1), steps + i)], 2)
        compare(o[:, :, i], q[:, :, i])


def batch(seed=4, lens=(900, 5, 0, 300, 64, 1200), prefix=256):
    B, Hq, Hkv, d, dd, w, ps = len(lens), 8, 2, 64, 16, 32, 64
    g = torch.Generator().manual_seed(seed)
    maxb = max(lens) // ps + 2
    shared = prefix // ps
    c = dar.DarPagedCache(B, Hkv, d, dd, w, ps, maxb, shared + B * maxb, BF)
    for t in (c.k_win, c.v_win, c.k_pool, c.v_pool):
        t.copy_(torch.randn(t.shape, generator=g))
    bt = torch.arange(B * maxb).reshape(B, maxb) + shared
    bt[:, :shared] = torch.arange(shared)
    c.block_table.copy_(bt.to(torch.int32))
    c.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    q = (torch.randn(B, Hq, d, generator=g) * 2).to(BF).cuda()
    wd = (torch.randn(Hkv, d, dd, generator=g) / 8).to(BF).cuda()
    new = [torch.randn(B, Hkv, d, generator=g).to(BF).cuda() for _ in range(2)]
    scores = torch.rand(B, Hkv, c.cap, generator=g).cuda()
    return c, q, wd, new, scores, c.block_table[0, :shared].clone()


def held(c, scores, *more):
    return [x.clone() for x in (c.k_win, c.v_win, c.k_pool, c.v_pool, c.lens, scores, *more)]


def restore(c, scores, saved):
    for t, x in zip((c.k_win, c.v_win, c.k_pool, c.v_pool, c.lens, scores), saved):
        t.copy_(x)


def same(a, b):
    return all(torch.equal(x.view(torch.int16) if x.dtype == BF else x.view(torch.int32),
                           y.view(torch.int16) if y.dtype == BF else y.view(torch.int32))
               for x, y in zip(a, b))


def sizes(c, q, n_prefix, n_keep):
    s = dar.make_shape(c.B, q.shape[1], c.Hkv, c.d, c.d_down, c.w, BF)
    return (dar.dar_decode_prefix_workspace_bytes(s, c.cap, n_prefix),
            dar.dar_cache_evict_workspace_bytes(s, c.cap, n_keep))


def step(c, q, wd, new, scores, blocks, o, ws=None, wse=None, stream=None):
    dar.dar_cache_append_paged(c, new[0], new[1], wd, Hq=q.shape[1], stream=stream)
    dar.dar_attn_decode_paged_scored(c, q, wd, scores, prefix_blocks=blocks, o=o, ws=ws, stream=stream)
    dar.dar_cache_evict_paged(c, scores, 400, n_fixed=256, ws=wse, stream=stream)


def test_captured_step():
    """One step captured and replayed, with eager steps of another batch that use
    the same workspaces between the replays: each replay ends where the eager
    step ended from the same state."""
    c, q, wd, new, scores, blocks = batch()
    start = held(c, scores)
    o = torch.empty_like(q)
    need = sizes(c, q, 256, 400)
    ws, wse = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in need)
    step(c, q, wd, new, scores, blocks, o, ws, wse)
    torch.cuda.synchronize()
    want = held(c, scores, o)
    other = batch(seed=5)
    o2 = torch.empty_like(q)
    graph, cs = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    restore(c, scores, start)
    cs.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(cs):
        with torch.cuda.graph(graph, stream=cs):
            step(c, q, wd, new, scores, blocks, o, ws, wse)
    torch.cuda.current_stream().wait_stream(cs)
    for rep in range(3):
        restore(c, scores, start)
        o.fill_(float("nan"))
        step(other[0], other[1], other[2], other[3], other[4], other[5], o2, ws, wse)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert same(held(c, scores, o), want), "replay %d" % rep


def test_two_graphs_one_workspace():
    """Two captured steps of different batches that share their workspaces, played
    one after the other."""
    ends, graphs = [], []
    users = [batch(seed=6), batch(seed=7, lens=(700, 1100, 301, 0, 1, 256 + 32))]
    outs = [torch.empty_like(u[1]) for u in users]
    needs = [sizes(u[0], u[1], 256, 400) for u in users]
    ws, wse = (torch.empty(max(n), dtype=torch.uint8, device="cuda") for n in zip(*needs))
    starts = [held(u[0], u[4]) for u in users]
    for u, o, s0 in zip(users, outs, starts):
        step(*u, o, ws, wse)
        torch.cuda.synchronize()
        ends.append(held(u[0], u[4], o))
        restore(u[0], u[4], s0)
        graph, cs = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        cs.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(cs):
            with torch.cuda.graph(graph, stream=cs):
                step(*u, o, ws, wse)
        torch.cuda.current_stream().wait_stream(cs)
        graphs.append(graph)
    for rep in range(3):
        for u, s0 in zip(users, starts):
            restore(u[0], u[4], s0)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for u, o, end in zip(users, outs, ends):
            assert same(held(u[0], u[4], o), end), rep


def test_another_stream():
    """Steps given a stream of their own, after work of the default stream on the
    same tensors; two batches on two streams at once."""
    users = [batch(seed=6), batch(seed=7)]
    outs = [torch.empty_like(u[1]) for u in users]
    starts = [held(u[0], u[4]) for u in users]
    ends = []
    for u, o, s0 in zip(users, outs, starts):
        step(*u, o)
        torch.cuda.synchronize()
        ends.append(held(u[0], u[4], o))
        restore(u[0], u[4], s0)
    spaces = [[torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes(u[0], u[1], 256, 400)]
              for u in users]
    streams = [torch.cuda.Stream() for _ in users]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for u, o, s, sp in zip(users, outs, streams, spaces):
        step(*u, o, *sp, stream=s)
    torch.cuda.synchronize()
    for u, o, end in zip(users, outs, ends):
        assert same(held(u[0], u[4], o), end)


def test_another_stream_with_its_own_memory():
    """The same with outputs and workspaces that the calls allocate, while the default
    stream goes on allocating and writing: what a call takes is not the default
    stream's."""
    users = [batch(seed=6), batch(seed=7)]
    starts = [held(u[0], u[4]) for u in users]
    ends = []

    def run(u, stream=None):
        c, q, wd, new, scores, blocks = u
        dar.dar_cache_append_paged(c, new[0], new[1], wd, Hq=q.shape[1], stream=stream)
        o = dar.dar_attn_decode_paged_scored(c, q, wd, scores, prefix_blocks=blocks, stream=stream)
        dar.dar_cache_evict_paged(c, scores, 400, n_fixed=256, stream=stream)
        return o, dar.dar_attn_decode_paged_prefix(c, q, wd, blocks, stream=stream)

    for u, s0 in zip(users, starts):
        outs = run(u)
        torch.cuda.synchronize()
        ends.append(held(u[0], u[4], *outs))
        restore(u[0], u[4], s0)
    streams = [torch.cuda.Stream() for _ in users]
    torch.cuda.synchronize()
    need = [n for u in users for n in sizes(u[0], u[1], 256, 400)]
    got, busy = [], []
    for u, s in zip(users, streams):
        got.append(run(u, s))
        # what the default stream would be given again, had it been its own
        for n in need:
            busy.append(torch.full((n,), 0xff, dtype=torch.uint8, device="cuda"))
            del busy[:-4]
    torch.cuda.synchronize()
    for u, outs, end in zip(users, got, ends):
        assert same(held(u[0], u[4], *outs), end)
