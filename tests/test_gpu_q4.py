"""4-bit weights with group scales: the layout byte for byte, and the product against
64 bits within the bound of its roundings, on pages of many sizes, CU masks, streams and graphs."""
import numpy as np
import pytest

import paper_2407_13996_amd as sg
import q4_oracle as qo

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
DT = {sg.BF16: torch.bfloat16, sg.F16: torch.float16}


@pytest.fixture(scope="module")
def ctx():
    c = sg.Context(0)
    yield c
    c.close()


class Matrix:
    """Random codes, scales and zero points on the host, and a pool with a page table for them."""

    def __init__(self, rows, cols, group, dtype, zeros, shift, seed=0, negative=False):
        rng, g = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
        self.group, self.dtype, self.shift = group, dtype, shift
        self.q = sg.q4(rows, cols, group, dtype, zeros)
        self.codes = rng.integers(0, 16, (rows, cols), dtype=np.uint8)
        s = 0.002 + 0.01 * torch.rand(rows, cols // group, generator=g)
        if negative:
            s = s * torch.where(torch.rand(s.shape, generator=g) < 0.5, -1, 1)
        self.scales = s.to(DT[dtype])
        self.zeros = torch.randint(0, 16, s.shape, generator=g).to(DT[dtype]) if zeros else None
        n = -(-sg.q4_bytes(self.q) >> shift)
        self.pages = n + n // 2 + 3
        self.table = torch.randperm(self.pages, generator=g)[:n].to(torch.int32)
        self.before = torch.randint(0, 256, (self.pages << shift,), generator=g, dtype=torch.uint8)

    def upload(self, ctx, stream=None):
        self.pool, self.d_table = self.before.to(DEV), self.table.to(DEV)
        self.w = sg.paged(self.pool, self.d_table, self.pages)
        codes = torch.from_numpy(self.codes).to(DEV)
        sg.colored_q4_pack(ctx, self.w, self.q, codes, self.scales.to(DEV),
                           None if self.zeros is None else self.zeros.to(DEV), self.shift, stream)
        return self

    def expect(self):
        bits = [None if t is None else t.view(torch.int16).numpy().view(np.uint16) for t in (self.scales, self.zeros)]
        whole = qo.packed(self.codes, *bits, self.group)
        assert len(whole) == sg.q4_bytes(self.q)
        pool = self.before.numpy().copy().reshape(self.pages, -1)
        size = 1 << self.shift
        for i, p in enumerate(self.table.tolist()):
            part = whole[i * size:(i + 1) * size]
            pool[p, :len(part)] = part
        return pool.reshape(-1)


SHAPES = [(1, 32, 32, sg.BF16, False, 10), (16, 128, 128, sg.F16, True, 10), (17, 160, 32, sg.F16, True, 12),
          (40, 192, 64, sg.BF16, True, 10), (33, 1152, 128, sg.BF16, False, 11), (100, 1056, 32, sg.BF16, False, 16)]


@pytest.mark.parametrize("rows,cols,group,dtype,zeros,shift", SHAPES)
def test_layout(ctx, rows, cols, group, dtype, zeros, shift):
    m = Matrix(rows, cols, group, dtype, zeros, shift).upload(ctx)
    torch.cuda.synchronize()
    assert np.array_equal(m.pool.cpu().numpy(), m.expect())
    assert ctx.device_error() == 0


def test_layout_from_a_slice_of_wider_rows(ctx):
    m = Matrix(21, 64, 32, sg.F16, False, 10)
    m.upload(ctx)
    wide = torch.full((21, 77), 255, dtype=torch.uint8)
    wide[:, 5:69] = torch.from_numpy(m.codes) | 0xA0      # upper bits do not count
    m.pool.copy_(m.before.to(DEV))
    sg.colored_q4_pack(ctx, m.w, m.q, wide.to(DEV)[:, 5:69], m.scales.to(DEV), None, m.shift)
    torch.cuda.synchronize()
    assert np.array_equal(m.pool.cpu().numpy(), m.expect())


def check(m, x, y):
    want, bound = qo.product(m.codes, m.scales, m.zeros, m.group, x)
    err = (y.cpu().double() - want).abs()
    assert bool((err <= bound + 1e-30).all()), float((err / bound).max())
    return float((err / bound).max())


def inputs(m, batch, seed=1):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(batch, m.q.cols, generator=g).to(DT[m.dtype])


@pytest.mark.parametrize("batch", [1, 3, 16])
@pytest.mark.parametrize("rows,cols,group,dtype,zeros,shift", SHAPES + [
    (1, 65536, 128, sg.BF16, True, 12), (5000, 384, 64, sg.F16, False, 13), (512, 4096, 128, sg.BF16, False, 21),
    (300, 11008, 32, sg.BF16, True, 14), (2000, 8192, 64, sg.F16, True, 16), (2500, 128, 32, sg.BF16, False, 10)])
def test_product(ctx, rows, cols, group, dtype, zeros, shift, batch):
    m = Matrix(rows, cols, group, dtype, zeros, shift, seed=rows + cols, negative=True).upload(ctx)
    x = inputs(m, batch)
    y = torch.full((batch + 1, rows), 7.0, device=DEV)
    sg.colored_gemv_q4(ctx, m.w, m.q, x.to(DEV), batch, y, m.shift)
    check(m, x, y[:batch])
    assert bool((y[batch] == 7.0).all())
    assert ctx.device_error() == 0


def test_same_bits_on_any_cus(ctx):
    """All CUs, whole XCDs, single CUs: the sums' order is the shape's."""
    for rows, cols in ((777, 1408), (4096, 4096)):
        m = Matrix(rows, cols, 64, sg.BF16, True, 14, seed=3).upload(ctx)
        x = inputs(m, 7).to(DEV)
        ys = []
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        for cus in (None, range(64), range(32, 224), [0, 5, 40, 41, 200], [17]):
            sg.set_cu_mask(ctx, s, cus)
            ys.append(torch.full((7, rows), -1.0, device=DEV))
            s.wait_stream(torch.cuda.current_stream())
            sg.colored_gemv_q4(ctx, m.w, m.q, x, 7, ys[-1], m.shift, stream=s)
        s.synchronize()
        sg.stream_release(ctx, s)
        check(m, x.cpu(), ys[0])
        for y in ys[1:]:
            assert torch.equal(y, ys[0])


def test_a_page_outside_the_pool_counts_as_zeros(ctx):
    """The first column segments of some rows, then a page of scales."""
    m = Matrix(64, 256, 32, sg.BF16, True, 10, seed=5).upload(ctx)
    x = inputs(m, 2)
    bad = m.table.clone()
    bad[2] = m.pages                     # block 2: rows 16..31, columns 0..127
    d_bad = bad.to(DEV)
    y = torch.zeros(2, 64, device=DEV)
    sg.colored_gemv_q4(ctx, sg.paged(m.pool, d_bad, m.pages), m.q, x.to(DEV), 2, y, m.shift)
    torch.cuda.synchronize()
    assert ctx.device_error() == sg.DEVERR_PT_RANGE
    cut = x.clone()
    cut[:, :128] = 0
    want, bound = qo.product(m.codes, m.scales, m.zeros, 32, x)
    part, _ = qo.product(m.codes, m.scales, m.zeros, 32, cut)
    want[:, 16:32] = part[:, 16:32]
    assert bool(((y.cpu().double() - want).abs() <= bound).all())
    bad = m.table.clone()
    bad[8] = -1                          # the first kilobyte of scales: all blocks'
    d_bad = bad.to(DEV)
    sg.colored_gemv_q4(ctx, sg.paged(m.pool, d_bad, m.pages), m.q, x.to(DEV), 2, y, m.shift)
    torch.cuda.synchronize()
    assert ctx.device_error() == sg.DEVERR_PT_RANGE
    assert bool((y == 0).all())


def test_rows_that_are_not_finite_stay_apart(ctx):
    m = Matrix(50, 384, 128, sg.BF16, False, 12, seed=6).upload(ctx)
    x = inputs(m, 4)
    x[1, 200], x[2, 5] = float("inf"), float("nan")
    y = torch.zeros(4, 50, device=DEV)
    sg.colored_gemv_q4(ctx, m.w, m.q, x.to(DEV), 4, y, m.shift)
    assert bool(torch.isnan(y[1:3]).all())
    good = torch.stack([x[0], x[3]])
    check(m, good, y[[0, 3]])


def test_matrix_past_4_gib(ctx):
    """Pages whose addresses pass 32 bits, the tensor's own bytes past them too."""
    rows, cols, group, shift = 140000, 65536, 128, 21
    q = sg.q4(rows, cols, group, sg.F16)
    n = -(-sg.q4_bytes(q) >> shift)
    pool = torch.zeros(n << shift, dtype=torch.uint8, device=DEV)
    table = torch.arange(n, dtype=torch.int32, device=DEV).flip(0).contiguous()
    tiles, segs, per = qo.sizes(rows, cols, group)
    # scales of 1 in the last tile and in row 0, codes random there
    whole = pool.view(n, 1 << shift).flip(0)          # the tensor in its own order (a copy)
    flat = whole.flatten()
    g = torch.Generator(device=DEV).manual_seed(2)
    picked = [0, 8749]
    for t in picked:
        flat[t * segs * 1024:(t + 1) * segs * 1024] = torch.randint(0, 256, (segs * 1024,), generator=g, device=DEV,
                                                                    dtype=torch.uint8)
        at = tiles * segs * 1024 + t * segs * per * 32
        flat[at:at + segs * per * 32].view(torch.float16).fill_(1.0)
    pool.copy_(flat.view(n, -1).flip(0).flatten())
    x = torch.randn(1, cols, generator=g, device=DEV).to(torch.float16)
    y = torch.full((1, rows), 9.0, device=DEV)
    sg.colored_gemv_q4(ctx, sg.paged(pool, table, n), q, x, 1, y, shift)
    y = y.cpu()
    assert bool((y[0, 16:8749 * 16] == 0).all())
    for t in picked:
        b = flat[t * segs * 1024:(t + 1) * segs * 1024].cpu().numpy().reshape(segs, 4, 16, 4, 4)
        nib = np.stack([b & 15, b >> 4], -1).reshape(segs, 4, 16, 4, 8)[..., [0, 4, 1, 5, 2, 6, 3, 7]]
        codes = nib.transpose(2, 0, 3, 1, 4).reshape(16, cols)
        want, bound = qo.product(codes, torch.ones(16, cols // group), None, group, x.cpu())
        got = y[:, t * 16:t * 16 + 16]
        rows_here = got.shape[1]
        assert bool(((got.double() - want[:, :rows_here]).abs() <= bound[:, :rows_here]).all())
    assert ctx.device_error() == 0


def test_captured_and_replayed(ctx):
    """A graph of a layout and a product, replayed with other inputs between eager calls."""
    m = Matrix(200, 512, 64, sg.BF16, False, 13, seed=8).upload(ctx)
    codes, scales = torch.from_numpy(m.codes).to(DEV), m.scales.to(DEV)
    x = inputs(m, 5).to(DEV)
    y = torch.zeros(5, 200, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        sg.colored_gemv_q4(ctx, m.w, m.q, x, 5, y, m.shift)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        sg.colored_q4_pack(ctx, m.w, m.q, codes, scales, None, m.shift)
        sg.colored_gemv_q4(ctx, m.w, m.q, x, 5, y, m.shift)
    for i in range(4):
        new = inputs(m, 5, seed=20 + i)
        x.copy_(new)
        m.codes = np.random.default_rng(i).integers(0, 16, m.codes.shape, dtype=np.uint8)
        codes.copy_(torch.from_numpy(m.codes))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(m, new, y)
        again = torch.zeros_like(y)
        sg.colored_gemv_q4(ctx, m.w, m.q, x, 5, again, m.shift)
        torch.cuda.synchronize()
        assert torch.equal(again, y)
    sg.stream_release(ctx, s)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [sg.BF16, sg.F16])
def test_same_bits_in_every_form(ctx, dtype, group, zeros):
    """Fewer CUs have tiles of more rows, and small batches x in LDS: the number of
    row blocks a CU has passes every bound of that choice, on whole XCDs and on parts."""
    s = torch.cuda.Stream()
    for rows, cols, batches in ((999, 1152, (1, 2, 3, 16)), (3300, 1152, (1, 6)), (2500, 256, (1, 16))):
        m = Matrix(rows, cols, group, dtype, zeros, 13, seed=rows + group, negative=True).upload(ctx)
        for batch in batches:
            x = inputs(m, batch, seed=batch)
            d_x, ys = x.to(DEV), []
            for cus in (None, range(64), range(32), range(16), range(3, 7), [200]):
                sg.set_cu_mask(ctx, s, cus)
                ys.append(torch.full((batch, rows), -1.0, device=DEV))
                s.wait_stream(torch.cuda.current_stream())
                sg.colored_gemv_q4(ctx, m.w, m.q, d_x, batch, ys[-1], m.shift, stream=s)
            s.synchronize()
            check(m, x, ys[0])
            assert all(torch.equal(y, ys[0]) for y in ys[1:])
    sg.stream_release(ctx, s)
    assert ctx.device_error() == 0


def test_pack_on_any_cus(ctx):
    m = Matrix(1003, 1056, 32, sg.F16, True, 12, seed=9).upload(ctx)
    want = m.expect()
    codes, scales, zeros = torch.from_numpy(m.codes).to(DEV), m.scales.to(DEV), m.zeros.to(DEV)
    s = torch.cuda.Stream()
    for cus in (None, range(64), range(5, 40), [17]):
        sg.set_cu_mask(ctx, s, cus)
        m.pool.copy_(m.before)
        s.wait_stream(torch.cuda.current_stream())
        sg.colored_q4_pack(ctx, m.w, m.q, codes, scales, zeros, m.shift, stream=s)
        s.synchronize()
        assert np.array_equal(m.pool.cpu().numpy(), want)
    sg.stream_release(ctx, s)
