"""Rotated cache writes of so many tokens that a tile holds several heads, and their values come in tiles of 32:
against the formula in 64 bits, on the device; V and all that is not written bit for bit.  A tile's heads leave remainders
of the four that are on their way at a time, and the last tile of a token has fewer than the others."""
import pytest

import kv_oracle as ko
import paper_2407_13996_amd as sg
from test_gpu_kv_rotate import DT, Call, turned

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = sg.Context(0)
    yield c
    c.close()


def ceil(a, b):
    return -(-a // b)


def tiles(n, heads, kv, dim):
    """(tiles, most heads of one, tokens of a tile of values) of a call: heads are put together while
    there are more than 2048 tiles of rows, values come 16 tokens a tile up to 2048 of those."""
    groups = ceil(n, 256 // {64: 4, 96: 8, 128: 8, 256: 16}[dim])
    most = min(heads + kv, ceil(groups * (heads + kv), 2048))
    sizes = [ceil(h, ceil(h, most)) for h in (heads, kv)]
    tokens = 16 if ceil(n, 16) * kv <= 2048 else 32
    return groups * (ceil(heads, sizes[0]) + ceil(kv, sizes[1])) + ceil(n, tokens) * kv, sizes, tokens


def slots_at(block, heads, dim, page_elems, index, slots):
    """Element indices of K or V at token slots, on the device."""
    s = slots[:, None, None]
    h, d = torch.arange(heads, device=DEV)[:, None], torch.arange(dim, device=DEV)
    return index(page_elems, block, dim, s // block, s % block, h, d)


def near(got, want, err, dtype):
    bound = err + ko.ROUND[dtype] * (want.abs() + err) + 2.0 ** -25
    worst = float(((got.double() - want).abs() / bound).max())
    assert worst <= 1.0, worst


def check(c, ctx, in_place, eps=1e-5):
    """As Call.check, with the 64-bit formula on the device, some tokens at a time."""
    torch.cuda.synchronize()
    assert ctx.device_error() == 0
    dt, proj = DT[c.dtype], c.proj.to(DEV)
    dev = [None if t is None else t.to(DEV) for t in (c.position, c.freq, c.q_norm, c.k_norm, c.slots)]
    position, freq, q_norm, k_norm, slots = dev
    q, k, v = c.parts(proj)
    before = q if in_place else torch.full(q.shape, 3.0, dtype=dt, device=DEV)
    per, mine = 1 << (c.shift - 1), c.pool.to(DEV)
    here = c.d_pool.view(dt)
    for a in range(0, c.n, 2048):
        cut = slice(a, min(a + 2048, c.n))
        on = position[cut] >= 0
        want, err = turned(q[cut], position[cut], freq, q_norm, eps, c.pairs)
        near(c.out[cut][on], want[on], err[on], dt)
        assert torch.equal(c.out[cut][~on].view(torch.int16), before[cut][~on].view(torch.int16))
        ok = on & (slots[cut] >= 0)
        at = slots_at(c.block, c.kv, c.dim, per, ko.k_index, slots[cut][ok])
        want, err = turned(k[cut], position[cut], freq, k_norm, eps, c.pairs)
        near(here[at], want[ok], err[ok], dt)
        mine[at] = c.d_pool[at]
        at = slots_at(c.block, c.kv, c.dim, per, ko.v_index, slots[cut][ok])
        mine[at] = v[cut][ok].contiguous().view(torch.int16)
    assert torch.equal(c.d_pool, mine)            # V, and all that is not written
    first = c.heads if in_place else 0
    assert torch.equal(c.d_proj[:, first:].contiguous().view(torch.int16), proj[:, first:].contiguous().view(torch.int16))


# n, heads, kv, dim, block, dtype, rot, pairs, norm, in place, CUs
CASES = [(5000, 15, 5, 96, 32, sg.F16, 64, True, "qk", False, None),
         (9000, 14, 2, 128, 16, sg.BF16, 128, False, "q", True, None),
         (2500, 40, 8, 256, 16, sg.BF16, 256, False, "k", False, range(64)),
         (2700, 21, 7, 256, 32, sg.F16, 128, True, "", True, None),
         (4200, 40, 8, 256, 32, sg.F16, 192, True, "qk", False, None),
         (10300, 48, 4, 64, 32, sg.F16, 64, False, "q", True, range(96)),
         (18000, 64, 8, 64, 16, sg.BF16, 64, True, "qk", False, None),
         (1100, 32, 32, 64, 16, sg.F16, 32, False, "k", False, [3, 40, 41, 170]),
         (1100, 32, 32, 64, 64, sg.BF16, 0, False, "q", True, None),
         (1111, 32, 32, 96, 16, sg.BF16, 96, True, "qk", False, None),
         (1090, 64, 32, 96, 64, sg.F16, 48, False, "", True, range(5, 77)),
         (8100, 5, 5, 128, 64, sg.F16, 128, True, "qk", False, range(32, 224)),
         (4321, 24, 8, 128, 32, sg.BF16, 64, False, "qk", False, None),
         (1081, 32, 32, 256, 16, sg.F16, 256, False, "q", False, None),
         (1065, 62, 31, 256, 16, sg.BF16, 64, True, "k", True, None)]


def test_the_cases_reach_what_they_say():
    """Heads a tile from one to ten: below four, remainders of one, two and three, fewer in the last tile of queries
    and of keys; tiles of 32 values for every head size and type."""
    found, wide, short = set(), set(), set()
    for n, heads, kv, dim, _, dtype, *_ in CASES:
        _, sizes, tokens = tiles(n, heads, kv, dim)
        found |= {s if s < 4 else s % 4 + 4 for s in sizes}
        short |= {i for i, h in enumerate((heads, kv)) if h % sizes[i]}
        if tokens == 32:
            wide.add((dim, dtype))
    assert found == {1, 2, 3, 4, 5, 6, 7} and short == {0, 1}, (found, short)
    assert wide == {(d, t) for d in (64, 96, 128, 256) for t in (sg.BF16, sg.F16)}, wide


@pytest.mark.parametrize("n,heads,kv,dim,block,dtype,rot,pairs,norm,in_place,cus", CASES)
def test_many_heads_a_tile(ctx, n, heads, kv, dim, block, dtype, rot, pairs, norm, in_place, cus):
    c = Call(n, heads, kv, dim, block, dtype, rot, pairs, norm, seed=dim)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    sg.set_cu_mask(ctx, s, cus)
    with torch.cuda.stream(s):
        c.run(ctx, in_place=in_place, stream=s)
    s.synchronize()
    assert ctx.last_tiles(s) == tiles(n, heads, kv, dim)[0]
    check(c, ctx, in_place)
    sg.stream_release(ctx, s)


def test_captured_in_place(ctx):
    """A graph that rotates queries in place, replayed on other rows with eager calls between: each replay gives
    the eager call's bits."""
    c = Call(3000, 30, 10, 128, 32, sg.BF16, 128, False, "qk")
    assert tiles(3000, 30, 10, 128)[1] == [2, 2]
    s = torch.cuda.Stream()
    c.run(ctx, in_place=True)
    torch.cuda.synchronize()
    q, k, v = c.parts(c.d_proj)
    dev = [t.to(DEV) for t in (c.slots, c.position, c.freq, c.q_norm, c.k_norm)]
    cache = sg.kv_cache(c.d_pool, c.pages, c.shift, c.block, c.kv, c.dim, c.dtype)

    def go():
        sg.colored_kv_append_rotated(ctx, cache, 0, q, k, v, q, dev[0], dev[1], freq=dev[2], q_norm=dev[3],
                                     k_norm=dev[4], eps=1e-5)

    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        go()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        go()
    for i in range(3):
        c.proj = torch.randn(c.proj.shape, generator=torch.Generator().manual_seed(i)).to(c.proj.dtype)
        got = []
        for call in (graph.replay, go):
            c.d_proj.copy_(c.proj)
            c.d_pool.copy_(c.pool)
            torch.cuda.synchronize()
            call()
            torch.cuda.synchronize()
            got.append((c.d_proj.clone(), c.d_pool.clone()))
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(*got))
        check(c, ctx, True)
    sg.stream_release(ctx, s)
