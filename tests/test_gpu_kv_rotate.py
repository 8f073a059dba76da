"""Cache writes with norms and rotation on the way, against the formula in 64 bits; V and all that is not
written bit for bit."""
import math

import pytest

import kv_oracle as ko
import paper_2407_13996_amd as sg

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
DT = {sg.BF16: torch.bfloat16, sg.F16: torch.float16}
E = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    c = sg.Context(0)
    yield c
    c.close()


def turned(x, position, freq, weight, eps, pairs):
    """The formula in 64 bits, and the bound of the kernel's error.

    A norm: a sum of dim squares in a tree (16 in a row, then at most 4 exchanges), its
    mean and root, the product with the weight: at most (20 + 6) / 2 + 5 roundings. An
    angle in turns keeps 53 bits, of which position takes up to 31 off the fraction; sine and
    cosine of the rest are off by 4 roundings of 1, the rest itself by one (pi of it in
    radians). A product and a sum more each; then one rounding to the type."""
    x = x.double()
    dim, err = x.shape[-1], torch.zeros_like(x)
    if weight is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * weight.double()
        err = 18 * E * x.abs()
    if freq is not None and len(freq):
        half = len(freq)
        i = torch.arange(half)
        a, b = (2 * i, 2 * i + 1) if pairs else (i, i + half)
        angle = position.double()[:, None, None] * freq.double()
        away = 8 * E + angle.abs() * 2.0 ** -51
        u, v, eu, ev = x[..., a], x[..., b], err[..., a], err[..., b]
        c, s = torch.cos(angle), torch.sin(angle)
        x, err = x.clone(), err.clone()
        x[..., a], x[..., b] = u * c - v * s, u * s + v * c
        err[..., a] = err[..., b] = eu + ev + (away + 2 * E) * (u.abs() + v.abs())
    return x, err


def close(got, want, err, dtype):
    off = (got.double() - want).abs()
    bound = err + ko.ROUND[dtype] * (want.abs() + err) + 2.0 ** -25
    assert bool((off <= bound).all()), float((off / bound).max())


def angles(half, scale=1.0):
    return (scale * 10000.0 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))).float()


class Call:
    def __init__(self, n, heads, kv, dim, block, dtype, rot, pairs, norm, norm_dtype=None, far=5000, seed=0, layers=1,
                 kind="runs"):
        g = torch.Generator().manual_seed(seed + n)
        dt = DT[dtype]
        self.n, self.heads, self.kv, self.dim, self.block, self.dtype, self.pairs = n, heads, kv, dim, block, dtype, pairs
        self.proj = torch.randn(n, heads + 2 * kv + 1, dim, generator=g).to(dt)
        self.freq = angles(rot // 2) if rot else None
        nd = norm_dtype or dt
        self.q_norm = (1 + 0.2 * torch.randn(dim, generator=g)).to(nd) if "q" in norm else None
        self.k_norm = (1 + 0.2 * torch.randn(dim, generator=g)).to(nd) if "k" in norm else None
        if kind == "single":
            self.pages = n + 3
            slots = torch.randperm(self.pages, generator=g)[:n] * block + torch.randint(0, block, (n,), generator=g)
            position = torch.randint(0, far, (n,), generator=g)
        else:
            # runs that begin and end anywhere, -1 between them
            self.pages = 3 * (n // block + 12) + n // 3
            perm, slots, position, page = torch.randperm(self.pages, generator=g), [], [], 0
            while len(slots) < n:
                run = int(torch.randint(1, 3 * block, (), generator=g))
                off, at = int(torch.randint(0, block, (), generator=g)), int(torch.randint(0, far, (), generator=g))
                if page + (off + run) // block + 1 > self.pages:
                    run, slots = 0, slots + [-1] * (n - len(slots))
                    position += [7] * (n - len(position))
                slots += [int(perm[page + (off + i) // block]) * block + (off + i) % block for i in range(run)] + [-1]
                position += [at + i for i in range(run)] + [-1 if run % 2 else at + run]
                page += (off + run) // block + 1
            slots, position = torch.tensor(slots[:n]), torch.tensor(position[:n])
        self.slots, self.position = slots.long(), position.to(torch.int32)
        self.elems, self.shift = ko.pages_of(kv, dim, block, layers)
        self.layers = layers
        self.pool = torch.randint(-(1 << 15), 1 << 15, (self.pages << (self.shift - 1),), generator=g,
                                  dtype=torch.int32).to(torch.int16)

    def parts(self, proj):
        h, k = self.heads, self.kv
        return proj[:, :h], proj[:, h:h + k], proj[:, h + k:h + 2 * k]

    def run(self, ctx, in_place=False, layer=0, stream=None, eps=1e-5):
        self.d_proj, self.d_pool = self.proj.to(DEV), self.pool.to(DEV)
        q, k, v = self.parts(self.d_proj)
        self.out = q if in_place else torch.full(q.shape, 3.0, dtype=q.dtype, device=DEV)
        dev = [None if t is None else t.to(DEV) for t in (self.slots, self.position, self.freq, self.q_norm, self.k_norm)]
        cache = sg.kv_cache(self.d_pool, self.pages, self.shift, self.block, self.kv, self.dim, self.dtype, self.layers,
                            2 * self.elems if self.layers > 1 else 0)
        sg.colored_kv_append_rotated(ctx, cache, layer, q, k, v, self.out, dev[0], dev[1], freq=dev[2], q_norm=dev[3],
                                     k_norm=dev[4], eps=eps, interleaved=self.pairs, stream=stream)
        return self

    def check(self, ctx, flag=0, layer=0, in_place=False, eps=1e-5):
        torch.cuda.synchronize()
        assert ctx.device_error() == flag
        q, k, v = self.parts(self.proj)
        dt = DT[self.dtype]
        on = self.position >= 0
        want, err = turned(q, self.position, self.freq, self.q_norm, eps, self.pairs)
        got = self.out.cpu()
        close(got[on], want[on], err[on], dt)
        before = q if in_place else torch.full(q.shape, 3.0, dtype=dt)
        assert torch.equal(got[~on].view(torch.int16), before[~on].view(torch.int16))
        ok = on & (self.slots >= 0) & (self.slots < self.pages * self.block)
        per, at = 1 << (self.shift - 1), self.slots[ok]
        pool, mine = self.d_pool.cpu(), self.pool.clone()
        here = pool[layer * self.elems:] if layer else pool
        there = mine[layer * self.elems:] if layer else mine
        rows = ko.rows(here, ko.k_index, per, self.block, self.kv, self.dim, at)
        want, err = turned(k, self.position, self.freq, self.k_norm, eps, self.pairs)
        close(rows.contiguous().view(dt), want[ok], err[ok], dt)
        ko.put_rows(there, ko.k_index, per, self.block, self.kv, self.dim, at, rows)
        ko.put_rows(there, ko.v_index, per, self.block, self.kv, self.dim, at, v[ok].contiguous().view(torch.int16))
        assert torch.equal(pool, mine)
        # the rest of the projection is as it was
        rest = self.d_proj.cpu()[:, self.heads if in_place else 0:]
        assert torch.equal(rest.contiguous().view(torch.int16),
                           self.proj[:, self.heads if in_place else 0:].contiguous().view(torch.int16))


@pytest.mark.parametrize("n,heads,kv,dim,block,dtype,rot,pairs,norm,kind", [
    (1, 8, 1, 64, 16, sg.BF16, 64, False, "qk", "single"), (61, 32, 8, 128, 64, sg.BF16, 128, False, "qk", "single"),
    (17, 6, 2, 96, 32, sg.F16, 96, False, "", "runs"), (130, 4, 4, 96, 16, sg.F16, 64, True, "k", "runs"),
    (33, 8, 8, 256, 64, sg.BF16, 256, False, "q", "runs"), (250, 14, 2, 64, 128, sg.F16, 32, True, "qk", "runs"),
    (70, 3, 3, 128, 16, sg.BF16, 0, False, "qk", "runs"), (41, 5, 5, 256, 16, sg.F16, 16, False, "", "runs"),
    (900, 15, 5, 128, 64, sg.F16, 96, False, "qk", "runs"), (700, 64, 8, 64, 32, sg.BF16, 64, True, "", "runs"),
    (600, 16, 16, 96, 64, sg.BF16, 48, False, "qk", "runs"), (300, 40, 8, 256, 32, sg.F16, 256, True, "qk", "runs"),
    (9, 1, 1, 128, 1024, sg.BF16, 0, True, "", "runs")])
def test_rotated_writes(ctx, n, heads, kv, dim, block, dtype, rot, pairs, norm, kind):
    Call(n, heads, kv, dim, block, dtype, rot, pairs, norm, kind=kind).run(ctx).check(ctx)


@pytest.mark.parametrize("n", [40, 600])
def test_in_place(ctx, n):
    Call(n, 32, 4, 128, 32, sg.BF16, 128, False, "qk").run(ctx, in_place=True).check(ctx, in_place=True)


@pytest.mark.parametrize("norm_dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_types_of_the_norms_weights(ctx, norm_dtype):
    Call(50, 8, 2, 96, 16, sg.F16, 32, True, "qk", norm_dtype=norm_dtype).run(ctx).check(ctx)


def test_far_positions_keep_their_fraction(ctx):
    """Up to 2^31 - 1, and angles of several turns a position."""
    for pairs in (False, True):
        c = Call(64, 4, 2, 128, 16, sg.F16, 128, pairs, "", kind="single")
        c.position = torch.tensor([0, 1, 2, 100, 65535, 1 << 20, (1 << 24) + 1, (1 << 31) - 1] * 8, dtype=torch.int32)
        c.run(ctx).check(ctx)
        c.freq = angles(64, scale=37.5)
        c.freq[3] = -2.5
        c.freq[4] = 0.0
        c.position = (c.position.long() % (1 << 26)).to(torch.int32)
        c.run(ctx).check(ctx)


def test_what_does_not_turn_keeps_its_bits(ctx):
    """Without norms the dimensions past rot pass as they are, infinities too; a row of zeros with a norm
    stays zero with eps, and one element's infinity stays in its pair."""
    c = Call(48, 4, 2, 96, 16, sg.BF16, 32, False, "")
    c.proj[:, :, 40] = float("inf")
    c.proj[:, :, 90] = -0.0
    c.run(ctx)
    torch.cuda.synchronize()
    on = c.position >= 0
    assert torch.equal(c.out.cpu()[on][:, :, 32:].contiguous().view(torch.int16),
                       c.proj[on][:, :4, 32:].contiguous().view(torch.int16))
    c = Call(20, 4, 4, 64, 16, sg.F16, 64, True, "qk")
    c.proj[3] = 0
    c.run(ctx).check(ctx)
    c = Call(20, 4, 4, 64, 16, sg.F16, 64, False, "")
    c.position = torch.arange(1, 21, dtype=torch.int32)
    c.proj[5, 2, 7] = float("inf")
    c.run(ctx)
    q = c.out.cpu()
    assert torch.isfinite(q).sum() == q.numel() - 2 and not torch.isfinite(q[5, 2, [7, 39]]).any()


def test_slots_out_of_range_are_flagged(ctx):
    for n in (70, 900):
        c = Call(n, 16, 8, 64, 16, sg.BF16, 64, False, "k")
        c.slots[5], c.slots[33], c.position[33], c.position[5] = c.pages * 16, -2, 9, 9
        c.run(ctx).check(ctx, flag=sg.DEVERR_SEQ)
        c.position[5] = c.position[33] = -1           # padding: its slots mean nothing
        c.run(ctx)
        torch.cuda.synchronize()
        # (nothing of such a token is written, so nothing is out of range)
        c.check(ctx)


def test_layers_and_masks_and_streams(ctx):
    s = torch.cuda.Stream()
    for cus, layer in ((None, 0), (range(64), 1), ([1, 33, 65, 200], 2)):
        c = Call(333, 8, 2, 64, 16, sg.BF16, 64, False, "qk", layers=3)
        s.wait_stream(torch.cuda.current_stream())
        sg.set_cu_mask(ctx, s, cus)
        with torch.cuda.stream(s):
            c.run(ctx, layer=layer, stream=s)
        s.synchronize()
        c.check(ctx, layer=layer)
    sg.stream_release(ctx, s)


def test_captured_and_replayed(ctx):
    c = Call(90, 8, 2, 128, 32, sg.F16, 128, False, "qk")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    d_proj, d_pool = c.proj.to(DEV), c.pool.to(DEV)
    out = torch.full((90, 8, 128), 3.0, dtype=torch.float16, device=DEV)
    q, k, v = c.parts(d_proj)
    dev = [t.to(DEV) for t in (c.slots, c.position, c.freq, c.q_norm, c.k_norm)]
    cache = sg.kv_cache(d_pool, c.pages, c.shift, c.block, c.kv, c.dim, c.dtype)

    def go():
        sg.colored_kv_append_rotated(ctx, cache, 0, q, k, v, out, dev[0], dev[1], freq=dev[2], q_norm=dev[3],
                                     k_norm=dev[4], eps=1e-5)

    with torch.cuda.stream(s):
        go()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        go()
    for seed in range(3):
        new = Call(90, 8, 2, 128, 32, sg.F16, 128, False, "qk", seed=100 + seed)
        new.pages, new.shift = c.pages, c.shift
        new.slots = torch.where(new.slots >= c.pages * 32, -1, new.slots)
        new.pool = c.pool
        new.q_norm, new.k_norm = c.q_norm, c.k_norm
        d_proj.copy_(new.proj)
        d_pool.copy_(c.pool)
        out.fill_(3.0)
        dev[0].copy_(new.slots)
        dev[1].copy_(new.position)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        new.d_proj, new.d_pool, new.out = d_proj, d_pool, out
        new.check(ctx)
        first = out.clone()
        go()
        torch.cuda.synchronize()
        assert torch.equal(first, out)
    sg.stream_release(ctx, s)


def test_no_tokens(ctx):
    c = Call(1, 2, 1, 64, 16, sg.F16, 64, False, "")
    c.proj, c.slots, c.position, c.n = c.proj[:0], c.slots[:0], c.position[:0], 0
    c.run(ctx).check(ctx)
    assert math.prod(c.out.shape) == 0
