"""Layouts and products of 4-bit weights, rotated writes and draft verifications captured on a stream that the context has not
seen, without a call before: two graphs of one stream, replayed in turn with other inputs and eager
calls between, against the eager calls' bits and the host."""
import pytest

import paper_2407_13996_amd as sg
import test_gpu_draft_verify as tv
import test_gpu_kv_rotate as tr
import test_gpu_q4 as tq

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"


class Step:
    """Buffers of one graph, and the calls on them."""

    def __init__(self, ctx, seed, rows, n, counts, dtype):
        self.ctx, self.counts, self.dtype = ctx, counts, dtype
        self.m = m = tq.Matrix(rows, 1152, 64, sg.BF16, True, 13, seed=seed)
        m.pool, m.d_table = m.before.to(DEV), m.table.to(DEV)
        m.w = sg.paged(m.pool, m.d_table, m.pages)
        self.weights = [torch.from_numpy(m.codes).to(DEV), m.scales.to(DEV), m.zeros.to(DEV)]
        self.x = torch.zeros(5, 1152, dtype=torch.bfloat16, device=DEV)
        self.y = torch.zeros(5, rows, device=DEV)
        self.c = c = tr.Call(n, 8, 2, 128, 32, sg.BF16, 128, False, "qk", seed=seed)
        self.proj, self.pool = c.proj.to(DEV), c.pool.to(DEV)
        self.out = torch.zeros(n, 8, 128, dtype=torch.bfloat16, device=DEV)
        self.at = [t.to(DEV) for t in (c.slots, c.position, c.freq, c.q_norm, c.k_norm)]
        self.cache = sg.kv_cache(self.pool, c.pages, c.shift, c.block, c.kv, c.dim, c.dtype)
        self.host = tv.case(counts, 200001, "tree", dtype, seed)
        self.rows = [t.to(DEV) for t in self.host]
        k = len(counts)
        self.found = [torch.zeros(k, 16, dtype=torch.int32, device=DEV)] + [torch.zeros(k, dtype=torch.int32, device=DEV)
                                                                            for _ in range(2)]

    def go(self):
        ctx, m, c = self.ctx, self.m, self.c
        sg.colored_q4_pack(ctx, m.w, m.q, *self.weights, m.shift)
        sg.colored_gemv_q4(ctx, m.w, m.q, self.x, 5, self.y, m.shift)
        q, k, v = c.parts(self.proj)
        sg.colored_kv_append_rotated(ctx, self.cache, 0, q, k, v, self.out, self.at[0], self.at[1], freq=self.at[2],
                                     q_norm=self.at[3], k_norm=self.at[4], eps=1e-5)
        target, guess, *rest = self.rows
        sg.colored_draft_verify(ctx, target, *rest, *self.found, draft=guess)

    def set(self, seed):
        self.x.copy_(tq.inputs(self.m, 5, seed=seed))
        g = torch.Generator().manual_seed(seed)
        self.c.proj = torch.randn(self.proj.shape, generator=g).to(torch.bfloat16)
        self.proj.copy_(self.c.proj)
        self.host = tv.case(self.counts, 200001, "tree", self.dtype, seed)
        for b, t in zip(self.rows, self.host):
            b.copy_(t)
        self.clear()

    def clear(self):
        self.pool.copy_(self.c.pool)
        self.m.pool.copy_(self.m.before)
        self.out.fill_(3.0)
        self.y.fill_(-1.0)
        for t in self.found:
            t.fill_(77)
        torch.cuda.synchronize()

    def got(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.m.pool, self.y, self.out, self.pool, *self.found)]

    def check(self):
        tq.check(self.m, self.x.cpu(), self.y)
        self.c.d_proj, self.c.d_pool, self.c.out = self.proj, self.pool, self.out
        self.c.check(self.ctx)
        tv.compare(self.ctx, self.found, *self.host, path_stride=16)


def test_captured_first():
    ctx = sg.Context(0)
    try:
        s = torch.cuda.Stream()
        steps = [Step(ctx, 3, 900, 170, [5, 9], "f32"), Step(ctx, 4, 3000, 61, [3, 0, 12, 7], "bf16")]
        torch.cuda.synchronize()
        graphs = []
        for step in steps:
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=s):
                step.go()
        for seed in range(3):
            for step, graph in zip(steps, graphs):
                step.set(50 + seed)
                graph.replay()
                first = step.got()
                step.check()
                step.clear()
                step.go()
                assert all(torch.equal(a, b) for a, b in zip(first, step.got()))
        sg.stream_release(ctx, s)
    finally:
        ctx.close()
