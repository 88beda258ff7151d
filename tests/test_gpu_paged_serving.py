"""The paged calls together, as a server uses them: prompt chunks and decode
steps of several sequences (append, attention with mass), eviction, and more
steps on the shrunk cache; also captured into a HIP graph, on another stream,
and with two graphs in turn."""
import math

import numpy as np
import pytest

import paged_common as pc
import paper_2608_27875_amd as hyq
from oracle import paged_oracle as po

pytestmark = pytest.mark.gpu
D = 128
SCALE = 1 / math.sqrt(D)


class Server:
    """B sequences in one pool, with the oracle's values beside them."""

    def __init__(self, fmt="bf16", B=2, Hq=4, Hkv=2, page=16, pages=24, seed=0):
        import torch
        rng = self.rng = np.random.default_rng(seed)
        self.B, self.Hq, self.Hkv, self.page, self.fmt = B, Hq, Hkv, page, fmt
        self.n_pages = B * pages
        b, f = pc.FORMATS[fmt]
        self.cache = hyq.PagedCache(Hq=Hq, Hkv=Hkv, page=page, n_pages=self.n_pages, device="cuda",
                                    bits_kv=b, kv_format=f, mass=True)
        self.free = list(rng.permutation(self.n_pages))
        self.table = np.full((B, pages), -1, dtype=np.int32)
        self.lens, self.seen = [0] * B, [0] * B
        self.qw, self.kw = pc.bits(rng, D), pc.bits(rng, D)
        self.f = (1e4 ** -(np.arange(0, D, 2) / D)).astype(np.float32)
        self.rope = hyq.Rope(q_weight=pc.dev(self.qw), k_weight=pc.dev(self.kw), inv_freq=pc.dev(self.f))

    def room(self, b, n):
        need = -(-n // self.page)
        for i in range(need):
            if self.table[b, i] < 0:
                self.table[b, i] = self.free.pop()

    def values(self):
        """What the pages hold, as float64."""
        bufs = self.cache.bufs
        r = []
        for n in ("k", "v"):
            if self.fmt == "bf16":
                r.append(pc.host(bufs[n]))
            else:
                c = bufs[n].cpu().numpy()
                x = c.view(np.int8).astype(np.float64) if self.fmt == "int8" else po.orc.e4m3_decode(c)
                r.append(x * pc.host(bufs[n + "_scale"])[..., None])
        return r

    def step(self, news, check=True):
        import torch
        T = sum(news)
        cu = np.concatenate([[0], np.cumsum(news)])
        for b in range(self.B):
            self.room(b, self.lens[b] + news[b])
        raw = pc.bits(self.rng, T, self.Hq + 2 * self.Hkv, D)
        pos = np.concatenate([np.arange(s, s + n) for s, n in zip(self.seen, news)]).astype(np.int32)
        x = pc.dev(raw)
        q, k, v = x.split([self.Hq, self.Hkv, self.Hkv], dim=1)
        batch = pc.batch_of(cu, self.lens, self.table)
        q_out = torch.empty((T, self.Hq, D), dtype=torch.bfloat16, device="cuda")
        out = torch.empty((T, self.Hq, D), device="cuda")
        before = pc.host(self.cache.bufs["mass"])
        hyq.hyq_paged_append(self.cache, batch, self.rope, q, k, v, pc.dev(pos), q_out)
        hyq.hyq_paged_attn(self.cache, batch, q_out, out, mass=hyq.MASS_ADD,
                           ws=pc.workspace(self.cache, batch, True, T))
        torch.cuda.synchronize()
        kv, vv = self.values()
        if check:
            # the appended rows are those of the formula (8 bits: within a code step)
            want_k = po.norm_rope(po.bf16(raw)[:, self.Hq:self.Hq + self.Hkv], po.bf16(self.kw), pos, self.f, D)
            for b in range(self.B):
                for i in range(news[b]):
                    p, o = po.place(self.table, b, self.lens[b] + i, self.page, self.n_pages)
                    before[p, :, o] = 0.0
                    t = int(cu[b]) + i
                    top = np.abs(want_k[t]).max(-1, keepdims=True)
                    tol = 2.0 ** -8 * np.abs(want_k[t]) + 2.0 ** -17 * top if self.fmt == "bf16" else \
                        2.0 ** -4 * np.abs(want_k[t]) + top / 127
                    assert np.all(np.abs(kv[p, :, o] - want_k[t]) <= tol)
            qv = pc.host(q_out)
            mass = before
            want = po.attention(qv, kv, vv, cu, self.lens, self.table, self.Hkv, SCALE, mass, "add")
            e = pc.logit_error(qv, kv, SCALE)
            atol, rtol = pc.out_tolerance(qv, dict(k=kv, v=vv), SCALE, max(news) * self.Hq // self.Hkv, False)
            np.testing.assert_allclose(pc.host(out), want, rtol=rtol, atol=atol)
            np.testing.assert_allclose(pc.host(self.cache.bufs["mass"]), mass, rtol=2 * e + 2.0 ** -18)
        for b in range(self.B):
            self.lens[b] += news[b]
            self.seen[b] += news[b]
        return out

    def evict(self, budget, recent):
        import torch
        B, n = self.B, -(-budget // self.page)
        new_table = np.full_like(self.table, -1)
        for b in range(B):
            new_table[b, :n] = [self.free.pop() for _ in range(n)]
        mass, (kv, vv) = self.cache.bufs["mass"].cpu().numpy(), self.values()
        keep = torch.empty((B, self.Hkv, budget), dtype=torch.int32, device="cuda")
        new_lens = torch.empty((B,), dtype=torch.int32, device="cuda")
        hyq.hyq_evict(self.cache, pc.dev(np.array(self.lens, np.int32)), pc.dev(self.table),
                      pc.dev(new_table), keep, new_lens, max_len=max(self.lens), budget=budget, recent=recent)
        torch.cuda.synchronize()
        want, lens = po.evict(mass, self.lens, self.table, budget, recent)
        np.testing.assert_array_equal(keep.cpu().numpy(), want)
        np.testing.assert_array_equal(new_lens.cpu().numpy(), lens)
        k2, v2 = self.values()
        for b in range(B):
            for j in range(self.Hkv):
                for i in range(int(lens[b])):
                    p, o = po.place(self.table, b, int(want[b, j, i]), self.page, self.n_pages)
                    p2, o2 = po.place(new_table, b, i, self.page, self.n_pages)
                    assert np.array_equal(k2[p2, j, o2], kv[p, j, o])
                    assert np.array_equal(v2[p2, j, o2], vv[p, j, o])
            self.free += [int(p) for p in self.table[b] if p >= 0]
        self.table, self.lens = new_table, [int(x) for x in lens]


@pytest.mark.parametrize("fmt", ["bf16", "int8", "fp8"])
def test_serving_loop(fmt):
    s = Server(fmt, seed=len(fmt))
    s.step([70, 33])          # prompt chunks
    s.step([1, 40])           # a decode step beside a chunk
    for _ in range(3):
        s.step([1, 1])
    s.evict(40, 8)
    for _ in range(3):        # the shrunk cache goes on, positions too
        s.step([1, 1])
    s.step([3, 2])
    s.evict(40, 8)
    s.step([1, 1])


def test_in_a_hip_graph():
    """A step captured once and replayed with other lengths, tables, inputs; an
    eager program works between the replays; every replay equals the eager call."""
    import torch
    rng = np.random.default_rng(3)
    B, Hq, Hkv, page, pages = 3, 8, 2, 16, 20
    for max_new, T in ((1, 3), (40, 60)):
        bufs, _ = pc.pool(rng, "bf16", B * pages, Hkv, page)
        cache = pc.cache_of(bufs, "bf16", Hq, np.zeros((B * pages, Hkv, page), np.float32))
        table = torch.zeros((B, pages), dtype=torch.int32, device="cuda")
        cu = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
        lens = torch.zeros(B, dtype=torch.int32, device="cuda")
        new_table = torch.zeros((B, 2), dtype=torch.int32, device="cuda")
        pos = torch.zeros(T, dtype=torch.int32, device="cuda")
        x = torch.zeros((T, Hq + 2 * Hkv, D), dtype=torch.bfloat16, device="cuda")
        q, k, v = x.split([Hq, Hkv, Hkv], dim=1)
        q_out = torch.zeros((T, Hq, D), dtype=torch.bfloat16, device="cuda")
        out = torch.zeros((T, Hq, D), device="cuda")
        keep = torch.zeros((B, Hkv, 30), dtype=torch.int32, device="cuda")
        new_lens = torch.zeros(B, dtype=torch.int32, device="cuda")
        rope = hyq.Rope(inv_freq=pc.dev((1e4 ** -(np.arange(0, D, 2) / D)).astype(np.float32)))
        batch = hyq.PagedBatch(cu, lens, table, max_new=max_new, max_len=(pages - 3) * page - max_new)
        ws = pc.workspace(cache, batch, True, T)

        def step():
            hyq.hyq_paged_append(cache, batch, rope, q, k, v, pos, q_out)
            hyq.hyq_paged_attn(cache, batch, q_out, out, mass=hyq.MASS_ADD, ws=ws)
            hyq.hyq_evict(cache, lens, table[:, :pages], new_table, keep, new_lens, max_len=pages * page,
                          budget=30, recent=3)

        def fill(seed):
            r = np.random.default_rng(seed)
            n = [1] * B if max_new == 1 else [int(r.integers(0, 20)) for _ in range(B)]
            cu.copy_(pc.dev(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)))
            lens.copy_(pc.dev(r.integers(0, (pages - 3) * page - max_new, B).astype(np.int32)))
            perm = r.permutation(B * pages)
            table.fill_(-1)
            table[:, :pages - 2] = pc.dev(perm[:B * (pages - 2)].reshape(B, -1).astype(np.int32))
            new_table.copy_(pc.dev(perm[B * (pages - 2):].reshape(B, 2).astype(np.int32)))
            x.copy_(pc.dev(pc.bits(r, T, Hq + 2 * Hkv, D)))
            pos.copy_(pc.dev(r.integers(0, 1000, T).astype(np.int32)))
            for name in ("k", "v"):
                cache.bufs[name].copy_(pc.dev(bufs[name]))
            cache.bufs["mass"].fill_(0.25)
            out.fill_(5.0)
            q_out.fill_(5.0)
            keep.fill_(-1)

        def state():
            return [t.clone() for t in (out, q_out, keep, new_lens, *[cache.bufs[n] for n in ("k", "v", "mass")])]

        fill(0)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for seed in (1, 2, 3, 4):
            fill(seed)
            step()
            torch.cuda.synchronize()
            want = state()
            fill(seed)
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(state(), want):
                assert torch.equal(a, b)


def test_other_stream_and_views():
    """A stream of the caller's, handed over or current; inputs that are views
    with an offset and a token stride of their own."""
    import torch
    rng = np.random.default_rng(8)
    case = ([90, 20], [1, 30], 4, 2, 16, "bf16", 0, "none")
    bufs, vals = pc.pool(rng, "bf16", 12, 2, 16)
    table, _ = pc.tables(rng, [91, 50], 16)
    table = np.where((table < 0) | (table >= 12), 0, table)
    cu, lens = np.array([0, 1, 31]), [90, 20]
    q = pc.bits(rng, 31, 4, D)
    want = po.attention(po.bf16(q), vals["k"], vals["v"], cu, lens, table, 2, SCALE)
    cache = pc.cache_of(bufs, "bf16", 4)
    batch = pc.batch_of(cu, lens, table)
    big = torch.full((40, 4, D), float("nan"), device="cuda")
    qt = pc.dev(q)
    ws = pc.workspace(cache, batch, False, 31)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = big[5:36]
    hyq.hyq_paged_attn(cache, batch, qt, out, ws=ws, stream=side)
    side.synchronize()
    first = out.clone()
    big.fill_(float("nan"))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        hyq.hyq_paged_attn(cache, batch, qt, out, ws=ws)
    side.synchronize()
    assert torch.equal(first, out)
    assert torch.isnan(big[:5]).all() and torch.isnan(big[36:]).all()
    atol, rtol = pc.out_tolerance(po.bf16(q), vals, SCALE, 60, False)
    np.testing.assert_allclose(pc.host(out), want, rtol=rtol, atol=atol)
    # norm_rope of rows inside a wider tensor
    wide = pc.dev(pc.bits(rng, 6, 9, D))
    x = wide[:, 2:8]
    rope = hyq.Rope(rot_dim=0)
    Q = torch.empty((1, 4, 6, D), dtype=torch.bfloat16, device="cuda")
    K = torch.empty((1, 1, 6, D), dtype=torch.bfloat16, device="cuda")
    V = torch.empty_like(K)
    pos = torch.zeros(6, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    hyq.hyq_norm_rope(hyq.Shape(B=1, Hq=4, Hkv=1, L=6), rope, x[:, :4], x[:, 4:5], x[:, 5:], pos, Q, K, V,
                      stream=side)
    side.synchronize()
    assert torch.equal(Q[0].transpose(0, 1), x[:, :4]) and torch.equal(V[0, 0], x[:, 5])


def test_two_graphs_share_a_workspace_in_turn():
    """Replays of two captured steps that use one workspace, one after the other."""
    import torch
    rng = np.random.default_rng(12)
    bufs, vals = pc.pool(rng, "fp8", 30, 2, 16)
    cache = pc.cache_of(bufs, "fp8", 8, np.zeros((30, 2, 16), np.float32))
    work = []
    for lens, news in (([200], [1]), ([150], [30])):
        cu = np.array([0, news[0]])
        table, _ = pc.tables(rng, [lens[0] + news[0]], 16)
        table = np.where((table < 0) | (table >= 30), 0, table)
        q = pc.bits(rng, news[0], 8, D)
        batch = pc.batch_of(cu, lens, table)
        out = torch.empty((news[0], 8, D), device="cuda")
        want = po.attention(po.bf16(q), vals["k"], vals["v"], cu, lens, table, 2, SCALE)
        tol = pc.out_tolerance(po.bf16(q), vals, SCALE, 4 * news[0], False)
        work.append((batch, pc.dev(q), out, want, tol))
    ws = torch.empty(max(hyq.hyq_paged_ws_bytes(cache, w[0], True, w[1].shape[0]) for w in work),
                     dtype=torch.uint8, device="cuda")
    graphs = []
    for batch, q, out, _, _ in work:
        hyq.hyq_paged_attn(cache, batch, q, out, mass=hyq.MASS_SET, ws=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            hyq.hyq_paged_attn(cache, batch, q, out, mass=hyq.MASS_SET, ws=ws)
        graphs.append(g)
    for _ in range(3):
        for g, (_, _, out, want, (atol, rtol)) in zip(graphs, work):
            out.fill_(float("nan"))
            ws.fill_(255)
            g.replay()
            torch.cuda.synchronize()
            np.testing.assert_allclose(pc.host(out), want, rtol=rtol, atol=atol)
