"""The 4-bit product where every fp32 sum is exact: whole codes and zero points, scales that are powers of two, x of small
whole numbers, so that the result has to be equal and a column left out, counted twice or scaled by a
neighbour's group shows at any number of columns.  All forms of the kernel: row blocks a tile, units of a wavefront from
one to many with full and partial ends, x in LDS up to its most and from the L2."""
import pytest

import paper_2407_13996_amd as sg
import q4_oracle as qo
from test_gpu_q4 import DT, Matrix

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = sg.Context(0)
    yield c
    c.close()


def whole(rows, cols, group, dtype, zeros, shift, seed):
    """A matrix whose scales are 1/2, 1, 2 and their opposites.  A product with x of at most 2 in magnitude has sums of halves
    below cols * 15 * 2 * 2 <= 2^22, and a group's sums of whole numbers stay below 128 * 31 * 2: exact in fp32."""
    m = Matrix(rows, cols, group, dtype, zeros, shift, seed)
    g = torch.Generator().manual_seed(seed + 1)
    s = torch.tensor([0.5, 1.0, 2.0, -0.5, -1.0, -2.0])
    m.scales = s[torch.randint(0, 6, m.scales.shape, generator=g)].to(DT[dtype])
    return m


def numbers(batch, cols, dtype, seed):
    """-2, -1, 1 and 2: no column that could go missing without a trace."""
    g = torch.Generator().manual_seed(seed)
    return torch.tensor([-2.0, -1.0, 1.0, 2.0])[torch.randint(0, 4, (batch, cols), generator=g)].to(DT[dtype])


def exact(m, x):
    """y on the device in 64 bits."""
    n = torch.from_numpy(m.codes).to(DEV).double()
    wide = lambda t: t.to(DEV).double().repeat_interleave(m.group, 1)  # noqa: E731
    w = wide(m.scales) * (n - (8.0 if m.zeros is None else wide(m.zeros)))
    return x.to(DEV).double() @ w.t().contiguous()


def form(ctx, m, stream=None):
    """(row blocks a tile, units of a wavefront, whether the last one is partly filled) of the last call."""
    row_blocks, segs = -(-m.q.rows // 16), -(-m.q.cols // 128)
    found = [b for b in (1, 2, 4) if -(-row_blocks // b) == ctx.last_tiles(stream)]
    assert len(found) == 1, (row_blocks, ctx.last_tiles(stream))
    run, per = -(-segs // 8), 4 // found[0]
    return found[0], -(-run // per), run % per != 0


def product(ctx, m, x, stream=None):
    y = torch.full((x.shape[0] + 1, m.q.rows), -7.0, device=DEV)
    sg.colored_gemv_q4(ctx, m.w, m.q, x.to(DEV), x.shape[0], y, m.shift, stream=stream)
    (stream or torch.cuda.current_stream()).synchronize()
    assert bool((y[-1] == -7.0).all())
    return y[:-1]


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("rows,cols,group,dtype,shift", [
    (16, 65536, 128, sg.BF16, 12), (33, 65536, 32, sg.F16, 16), (17, 65504, 32, sg.BF16, 14), (100, 11008, 64, sg.F16, 10),
    (4096, 11008, 128, sg.BF16, 21), (700, 32832, 64, sg.BF16, 13)])
def test_many_columns(ctx, rows, cols, group, dtype, shift, zeros):
    m = whole(rows, cols, group, dtype, zeros, shift, seed=cols + rows).upload(ctx)
    for batch in (1, 3, 16):
        x = numbers(batch, cols, dtype, batch)
        assert torch.equal(product(ctx, m, x).double(), exact(m, x)), batch
    assert ctx.device_error() == 0


# rows, columns, batch; row blocks a tile on all CUs, units, a partial last unit
TWO = [(5120, 5376, 1, 2, 3, False), (4200, 4352, 2, 2, 3, True), (8192, 9600, 1, 2, 5, False),
       (4900, 8448, 1, 2, 5, True), (4170, 1152, 1, 2, 1, False), (8192, 2048, 6, 2, 1, False)]
FOUR = [(11008, 4096, 8, 4, 4, False), (14336, 2176, 16, 4, 3, False), (9216, 384, 16, 4, 1, False)]
ONE = [(2000, 4096, 16, 1, 1, False), (4096, 6400, 1, 1, 2, True), (3100, 11008, 4, 1, 3, True),
       (4096, 8192, 3, 1, 2, False), (2000, 2944, 1, 1, 1, True), (4000, 5120, 2, 1, 2, True)]


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("i", range(len(TWO + FOUR + ONE)))
def test_every_form(ctx, i, group, zeros):
    """On all CUs, where the named form runs, and on masks on which others do; one type or the other, of
    each form, group and kind of zero points both."""
    rows, cols, batch, blocks, units, partial = (TWO + FOUR + ONE)[i]
    dtype = (sg.BF16, sg.F16)[i % 2]
    s = torch.cuda.Stream()
    m = whole(rows, cols, group, dtype, zeros, 16, seed=rows + group).upload(ctx)
    x = numbers(batch, cols, dtype, cols)
    want = exact(m, x)
    torch.cuda.synchronize()
    for cus in (None, range(32), range(9, 100)):
        sg.set_cu_mask(ctx, s, cus)
        y = product(ctx, m, x, s)
        if cus is None:
            assert form(ctx, m, stream=s) == (blocks, units, partial)
        assert torch.equal(y.double(), want), cus
    sg.stream_release(ctx, s)
    assert ctx.device_error() == 0


def test_the_most_of_x_in_lds(ctx):
    """Two row blocks, groups of 32, zero points: 48 KiB of sums and scales and 24 KiB of x a workgroup."""
    m = whole(8192, 2048, 32, sg.BF16, True, 21, seed=11).upload(ctx)
    x = numbers(6, 2048, sg.BF16, 12)
    y = product(ctx, m, x)
    assert 2048 * 2 * 6 == 24576 and form(ctx, m)[0] == 2
    assert torch.equal(y.double(), exact(m, x))
    g = torch.Generator().manual_seed(13)
    x = torch.randn(6, 2048, generator=g).to(torch.bfloat16)
    want, bound = qo.product(m.codes, m.scales, m.zeros, 32, x)
    assert bool(((product(ctx, m, x).cpu().double() - want).abs() <= bound).all())


def test_columns_past_4_gib(ctx):
    """As the tensor's bytes pass 32 bits: the first and the last rows' codes, all columns, exactly."""
    rows, cols, group, shift = 140000, 65536, 128, 21
    q = sg.q4(rows, cols, group, sg.F16, True)
    n = -(-sg.q4_bytes(q) >> shift)
    pool = torch.zeros(n << shift, dtype=torch.uint8, device=DEV)
    table = torch.arange(n, dtype=torch.int32, device=DEV).flip(0).contiguous()
    tiles, segs, per = qo.sizes(rows, cols, group)
    g = torch.Generator().manual_seed(3)

    def put(at, data):
        """``data`` (bytes on the host) at byte ``at`` of the tensor, page after page."""
        done = 0
        while done < len(data):
            page, off = (at + done) >> shift, (at + done) & ((1 << shift) - 1)
            size = min(len(data) - done, (1 << shift) - off)
            base = ((n - 1 - page) << shift) + off
            pool[base:base + size] = data[done:done + size].to(DEV)
            done += size

    x = numbers(2, cols, sg.F16, 4)
    want = {}
    for t in (0, tiles - 1):
        codes = torch.randint(0, 16, (16, cols), generator=g, dtype=torch.uint8).numpy()
        s = torch.tensor([0.5, 1.0, -2.0])[torch.randint(0, 3, (16, cols // group), generator=g)].to(torch.float16)
        z = torch.randint(0, 16, s.shape, generator=g).to(torch.float16)
        bits = [v.view(torch.int16).numpy().view("uint16") for v in (s, z)]
        b = torch.from_numpy(qo.packed(codes, *bits, group))
        k, p = segs * 1024, segs * per * 32
        put(t * k, b[:k])
        put(tiles * k + t * p, b[k:k + p])
        put(tiles * (k + p) + t * p, b[k + p:])
        want[t] = qo.product(codes, s, z, group, x)[0]
    y = torch.full((2, rows), 9.0, device=DEV)
    sg.colored_gemv_q4(ctx, sg.paged(pool, table, n), q, x.to(DEV), 2, y, shift)
    y = y.cpu().double()
    assert bool((y[:, 16:(tiles - 1) * 16] == 0).all())
    for t, w in want.items():
        got = y[:, t * 16:t * 16 + 16]
        assert torch.equal(got, w[:, :got.shape[1]])
    assert ctx.device_error() == 0


@pytest.mark.parametrize("dtype,x_to,s_to", [(sg.F16, -24, 0), (sg.F16, 0, -23), (sg.BF16, -133, 0), (sg.BF16, 0, -126)])
def test_denormal_numbers_count(ctx, dtype, x_to, s_to):
    """x or the scales at the smallest that their type has: nothing is taken for zero."""
    for rows, cols, batch in ((100, 1024, 3), (5120, 5376, 1), (11008, 4096, 8)):
        m = whole(rows, cols, 64, dtype, True, 14, seed=5)
        m.scales = (m.scales.double() * 2.0 ** s_to).to(DT[dtype])
        m.upload(ctx)
        x = (numbers(batch, cols, dtype, 1).double() * 2.0 ** x_to).to(DT[dtype])
        assert bool((x != 0).all()) and bool((m.scales != 0).all())
        assert torch.equal(product(ctx, m, x).double(), exact(m, x)), (rows, cols, batch)
