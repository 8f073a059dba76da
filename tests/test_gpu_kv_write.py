"""Writes to the paged key/value cache: new tokens by slot map and accepted
paths of drafts, the whole pool compared bit for bit with the host's."""
import numpy as np
import pytest

import kv_oracle as ko
import paper_2407_13996_amd as sg

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
DT = {sg.BF16: torch.bfloat16, sg.F16: torch.float16}


@pytest.fixture(scope="module")
def ctx():
    c = sg.Context(0)
    yield c
    c.close()


def bits(n, gen):
    """Every 16-bit pattern may occur: the writes move bits."""
    return torch.randint(-(1 << 15), 1 << 15, (n,), generator=gen, dtype=torch.int32).to(torch.int16)


def cache_of(pool, pages, shift, block, heads, dim, dtype, layers=1, stride=0):
    return sg.kv_cache(pool, pages, shift, block, heads, dim, dtype, layers, stride)


def slots_of(kind, n, block, pages, rng):
    if kind == "single":  # a token a block, odd places
        return rng.permutation(pages)[:n] * block + rng.integers(0, block, n)
    # runs that begin and end inside groups of eight and blocks, some tokens nowhere
    perm, out, page = rng.permutation(pages), [], 0
    while len(out) < n:
        run, off = int(rng.integers(1, 3 * block)), int(rng.integers(0, block))
        span = -(-(off + run) // block)
        if page + span > pages:
            break
        for i in range(run):
            out.append(perm[page + (off + i) // block] * block + (off + i) % block)
        out += [-1] * int(rng.integers(0, 3))
        page += span
    return np.array((out + [-1] * n)[:n])


@pytest.mark.parametrize("heads,dim,block,dtype,n,kind", [
    (8, 128, 64, sg.BF16, 61, "single"), (1, 64, 16, sg.F16, 1, "single"), (2, 96, 16, sg.F16, 333, "runs"),
    (5, 128, 32, sg.BF16, 1000, "runs"), (3, 256, 128, sg.BF16, 777, "runs"), (1, 64, 1024, sg.F16, 2049, "runs"),
    (2, 256, 16, sg.F16, 17, "runs"), (4, 96, 64, sg.BF16, 16, "runs")])
def test_append(ctx, heads, dim, block, dtype, n, kind):
    rng, gen = np.random.default_rng(n), torch.Generator().manual_seed(n)
    pages = n + 3 if kind == "single" else 4 * n // block + 40
    elems, shift = ko.pages_of(heads, dim, block)
    pool = bits(pages << (shift - 1), gen)
    slots = torch.from_numpy(slots_of(kind, n, block, pages, rng).astype(np.int64))
    proj = bits(n * (2 * heads + 3) * dim, gen).view(n, 2 * heads + 3, dim)
    k, v = proj[:, 1:1 + heads], proj[:, heads + 2:2 * heads + 2]
    d_pool, d_proj = pool.to(DEV), proj.to(DEV).view(DT[dtype])
    cache = cache_of(d_pool, pages, shift, block, heads, dim, dtype)
    sg.colored_kv_append(ctx, cache, 0, d_proj[:, 1:1 + heads], d_proj[:, heads + 2:2 * heads + 2], slots.to(DEV))
    on = slots >= 0
    ko.put_rows(pool, ko.k_index, 1 << (shift - 1), block, heads, dim, slots[on], k[on])
    ko.put_rows(pool, ko.v_index, 1 << (shift - 1), block, heads, dim, slots[on], v[on])
    torch.cuda.synchronize()
    assert torch.equal(d_pool.cpu(), pool)
    assert ctx.device_error() == 0


def test_append_in_any_order_and_out_of_range(ctx):
    """Tokens in reverse, in shuffled order, and slots past the pool: those are skipped and flagged."""
    heads, dim, block, pages, n = 2, 64, 16, 12, 150
    gen = torch.Generator().manual_seed(5)
    elems, shift = ko.pages_of(heads, dim, block)
    for order in (torch.arange(n).flip(0), torch.randperm(n, generator=gen), torch.arange(n) ^ 1):
        pool = bits(pages << (shift - 1), gen)
        slots = order.clone()
        bad = torch.zeros(n, dtype=torch.bool)
        bad[3], bad[77] = True, True
        slots[3], slots[77] = pages * block, -2
        kv = bits(2 * n * heads * dim, gen).view(2, n, heads, dim)
        d_pool, d_kv = pool.to(DEV), kv.to(DEV).view(torch.float16)
        sg.colored_kv_append(ctx, cache_of(d_pool, pages, shift, block, heads, dim, sg.F16), 0, d_kv[0], d_kv[1],
                             slots.to(DEV))
        ko.put_rows(pool, ko.k_index, 1 << (shift - 1), block, heads, dim, slots[~bad], kv[0][~bad])
        ko.put_rows(pool, ko.v_index, 1 << (shift - 1), block, heads, dim, slots[~bad], kv[1][~bad])
        torch.cuda.synchronize()
        assert torch.equal(d_pool.cpu(), pool)
        assert ctx.device_error() == sg.DEVERR_SEQ


def test_append_past_4_gib_and_on_other_cus(ctx):
    """Pages far beyond 4 GiB; a mask of single CUs; a stream of its own."""
    heads, dim, block, dtype = 8, 128, 64, sg.BF16
    elems, shift = ko.pages_of(heads, dim, block)
    pages = (6 << 30) >> shift
    d_pool = torch.zeros(pages << (shift - 1), dtype=torch.int16, device=DEV)
    pages_used = torch.tensor([0, pages // 2, pages - 1, pages - 7])
    slots = (pages_used[:, None] * block + torch.arange(5, 5 + 40)).flatten()
    gen = torch.Generator().manual_seed(1)
    kv = bits(2 * len(slots) * heads * dim, gen).view(2, len(slots), heads, dim)
    d_kv, d_slots = kv.to(DEV).view(torch.bfloat16), slots.to(DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    sg.set_cu_mask(ctx, s, [1, 33, 65, 200])
    cache = cache_of(d_pool, pages, shift, block, heads, dim, dtype)
    sg.colored_kv_append(ctx, cache, 0, d_kv[0], d_kv[1], d_slots, stream=s)
    s.synchronize()
    sg.stream_release(ctx, s)
    per = 1 << (shift - 1)
    for p in range(4):
        page = d_pool[int(pages_used[p]) * per:][:per].cpu()
        want = torch.zeros_like(page)
        local = torch.arange(5, 45)
        ko.put_rows(want, ko.k_index, per, block, heads, dim, local, kv[0][40 * p:40 * p + 40])
        ko.put_rows(want, ko.v_index, per, block, heads, dim, local, kv[1][40 * p:40 * p + 40])
        assert torch.equal(page, want)
    assert int((d_pool != 0).sum()) <= 4 * 2 * 40 * heads * dim
    assert ctx.device_error() == 0


def commit_oracle(pool, layers, stride, per, block, heads, dim, table, lens, path, accepted):
    for r in range(len(lens)):
        for i in range(int(accepted[r])):
            a, b = int(lens[r]) + int(path[r, i]), int(lens[r]) + i
            sa = int(table[r, a // block]) * block + a % block
            sb = int(table[r, b // block]) * block + b % block
            for layer in range(layers):
                flat = pool[layer * stride:]
                for index in (ko.k_index, ko.v_index):
                    ko.put_rows(flat, index, per, block, heads, dim, [sb],
                                ko.rows(flat, index, per, block, heads, dim, [sa]))


@pytest.mark.parametrize("inside", [True, False])
@pytest.mark.parametrize("heads,dim,block,dtype,layers,nodes", [(8, 128, 64, sg.BF16, 2, 24), (1, 64, 16, sg.F16, 3, 9),
                                                                 (3, 96, 16, sg.BF16, 2, 64), (2, 256, 32, sg.F16, 1, 33)])
def test_commit(ctx, heads, dim, block, dtype, layers, nodes, inside):
    """Ascending paths of every kind, entries that stay and entries whose source
    is a later entry's destination among them, layers side by side in a page or apart."""
    rng, gen = np.random.default_rng(nodes), torch.Generator().manual_seed(nodes)
    n = 7
    elems, shift = ko.pages_of(heads, dim, block, layers if inside else 1)
    width = -(-(200 + nodes) // block)
    pages = n * width + 2
    stride = elems if inside else pages << (shift - 1)
    pool = bits((1 if inside else layers) * pages << (shift - 1), gen)
    table = rng.permutation(pages)[:n * width].reshape(n, width)
    lens = np.array([0, 1, 13, 16, 99, 200, 57])
    accepted = np.array([nodes, 0, 1, nodes // 2, 3, nodes - 1, 2])
    path = np.zeros((n, nodes), int)
    for r in range(n):
        path[r, :accepted[r]] = np.sort(rng.permutation(nodes)[:accepted[r]])
    path[4, :3], path[6, :2] = [0, 2, 3], [1, 2]
    d_pool = pool.to(DEV)
    out = torch.full((n,), -5, dtype=torch.int32, device=DEV)
    i32 = lambda a: torch.from_numpy(a.astype(np.int32)).to(DEV)  # noqa: E731
    cache = cache_of(d_pool, pages, shift, block, heads, dim, dtype, layers, 2 * stride)
    sg.colored_kv_commit(ctx, cache, i32(table), i32(lens), i32(path), i32(accepted), out)
    commit_oracle(pool, layers, stride, 1 << (shift - 1), block, heads, dim, table, lens, path, accepted)
    torch.cuda.synchronize()
    assert out.cpu().tolist() == (lens + accepted).tolist()
    assert torch.equal(d_pool.cpu(), pool)
    assert ctx.device_error() == 0


def test_commit_cuts_paths_that_are_out_of_range(ctx):
    heads, dim, block, pages = 1, 64, 16, 20
    elems, shift = ko.pages_of(heads, dim, block)
    pool = bits(pages << (shift - 1), torch.Generator().manual_seed(3))
    table = np.arange(18).reshape(6, 3)
    table[5, 2] = 1000  # a page that the pool does not have
    lens = np.array([10, 20, 5, -1, 40, 30])
    path = np.array([[0, 2, 2, 5], [1, 3, 40, 41], [-1, 0, 1, 2], [0, 1, 2, 3], [0, 1, 2, 7], [1, 2, 3, 4]])
    accepted = np.array([4, 4, 3, 2, 9, 3])
    good = np.array([2, 2, 0, 0, 4, 3])
    i32 = lambda a: torch.from_numpy(a.astype(np.int32)).to(DEV)  # noqa: E731
    d_pool, out = pool.to(DEV), torch.zeros(6, dtype=torch.int32, device=DEV)
    sg.colored_kv_commit(ctx, cache_of(d_pool, pages, shift, block, heads, dim, sg.F16), i32(table), i32(lens),
                         i32(path), i32(accepted), out)
    commit_oracle(pool, 1, 0, 1 << (shift - 1), block, heads, dim, table[:5], lens[:5], path[:5],
                  np.where(lens[:5] < 0, 0, good[:5]))
    # request 5: token 30 + 1 lies in the sound second block, 30 + 2 and on in the third: only the first entry moves
    commit_oracle(pool, 1, 0, 1 << (shift - 1), block, heads, dim, table[5:], lens[5:], path[5:], [1])
    torch.cuda.synchronize()
    assert out.cpu().tolist() == [12, 22, 5, -1, 44, 33]
    assert torch.equal(d_pool.cpu(), pool)
    assert ctx.device_error() == sg.DEVERR_SEQ | sg.DEVERR_PT_RANGE


def test_bindings_refuse_rows_that_do_not_fit(ctx):
    elems, shift = ko.pages_of(2, 64, 16)
    pool = torch.zeros(4 << (shift - 1), dtype=torch.float16, device=DEV)
    cache = cache_of(pool, 4, shift, 16, 2, 64, sg.F16)
    k = torch.zeros(5, 2, 64, dtype=torch.float16, device=DEV)
    slots = torch.zeros(5, dtype=torch.int64, device=DEV)
    for bad in (k[:4], k[:, :1], k.to(torch.bfloat16), k[..., ::2], k.view(5, 128)):
        with pytest.raises(ValueError):
            sg.colored_kv_append(ctx, cache, 0, bad, k, slots)
    with pytest.raises(ValueError):
        sg.colored_kv_append(ctx, cache, 0, k, k, slots.int())
    with pytest.raises(sg.SgdrcError):
        sg.colored_kv_append(ctx, cache, 1, k, k, slots)
    odd = torch.zeros(5 * 2 * 68, dtype=torch.float16, device=DEV).view(5, 2, 68)[..., :64]
    with pytest.raises(sg.SgdrcError):
        sg.colored_kv_append(ctx, cache, 0, odd, k, slots)
    sg.colored_kv_append(ctx, cache, 0, k[:0], k[:0], slots[:0])
