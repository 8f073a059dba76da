"""Commits of drafts that got no pages or only some of their tokens: nothing but
the request's own tokens moves, whatever its row of the table still names."""
import numpy as np
import pytest

import kv_oracle as ko
import paper_2407_13996_amd as sg
from test_gpu_kv_write import bits, cache_of, commit_oracle

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = sg.Context(0)
    yield c
    c.close()


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a).astype(np.int32))).to(DEV)


class State:
    def __init__(self, ctx, requests, width, pages, block):
        self.ctx, self.n, self.block = ctx, requests, block
        self.ring = i32(np.arange(pages))
        self.pos = torch.tensor([0, pages], dtype=torch.int64, device=DEV)
        self.held, self.lens = i32(np.zeros(requests)), i32(np.zeros(requests))
        self.table = i32(np.zeros((requests, width)))

    def map(self, new):
        n = max(int(np.maximum(new, 0).sum()), 1)
        pos, held, totals = (torch.empty_like(t) for t in (self.pos, self.held, self.lens))
        slots = torch.empty(n, dtype=torch.int64, device=DEV)
        sg.colored_kv_map(self.ctx, self.block, self.ring, self.pos, self.held, self.lens, i32(new), self.table, pos,
                          held, totals, i32(np.zeros(self.n + 1)), slots, i32(np.zeros(n)), i32(np.zeros(n)))
        self.pos, self.held = pos, held
        return totals, slots


def test_a_request_that_was_not_served_commits_nothing(ctx):
    """Request 0 ends and request 1 takes its pages; when request 0 begins again
    and finds too few pages, its row still names those of request 1."""
    heads, dim, block, pages = 2, 64, 16, 4
    elems, shift = ko.pages_of(heads, dim, block)
    pool = bits(pages << (shift - 1), torch.Generator().manual_seed(1))
    d_pool = pool.to(DEV)
    cache = cache_of(d_pool, pages, shift, block, heads, dim, sg.BF16)
    s = State(ctx, 2, 4, pages, block)
    s.lens, _ = s.map([40, 10])                 # pages 0, 1, 2 and 3
    s.lens, _ = s.map([-1, 0])                  # 0, 1 and 2 are free again
    s.lens, _ = s.map([0, 30])                  # request 1 takes 0 and 1
    s.lens, _ = s.map([10, 0])                  # request 0 takes 2
    assert s.table[0, :3].tolist() == [2, 1, 2] and s.table[1, :3].tolist() == [3, 0, 1]
    totals, slots = s.map([20, 5])              # no page for request 0; request 1 has room
    assert totals.tolist() == [10, 45] and bool((slots[:20] == -1).all())
    path, accepted = i32([[0, 7, 9, 11], [0, 2, 3, 4]]), i32([4, 3])
    out = i32([-1, -1])
    sg.colored_kv_commit(ctx, cache, s.table, s.lens, path, accepted, out, totals=totals)
    commit_oracle(pool, 1, 0, 1 << (shift - 1), block, heads, dim, s.table.cpu().numpy(), [10, 40],
                  path.cpu().numpy(), [0, 3])
    torch.cuda.synchronize()
    assert out.tolist() == [10, 43]
    assert torch.equal(d_pool.cpu(), pool)
    assert ctx.device_error() == sg.DEVERR_SEQ
    # its length is sound for the next step
    s.lens = out
    assert s.map([2, 0])[0].tolist() == [12, 43] and ctx.device_error() == 0


@pytest.mark.parametrize("layers", [1, 3])
def test_paths_are_cut_at_the_totals(ctx, layers):
    """Paths past the drafted tokens, of all of them, and totals that are no lengths."""
    heads, dim, block, pages, most = 1, 96, 16, 24, 6
    elems, shift = ko.pages_of(heads, dim, block)
    rng = np.random.default_rng(layers)
    pool = bits(layers * pages << (shift - 1), torch.Generator().manual_seed(layers))
    d_pool = pool.to(DEV)
    cache = cache_of(d_pool, pages, shift, block, heads, dim, sg.F16, layers, 2 * (pages << (shift - 1)))
    table = rng.permutation(pages)[:24].reshape(8, 3)
    lens = np.array([10, 10, 10, 10, 10, 0, 30, 47])
    totals = np.array([16, 15, 13, 10, 9, -1, 49, 48])  # the last: one token before the row's end
    path = np.tile([0, 2, 3, 4, 5, 7], (8, 1))
    path[7, 0] = 0
    accepted = np.array([5, 5, 5, 5, 0, 2, 3, 2])
    good = np.array([5, 4, 2, 0, 0, 0, 0, 1])
    out = i32(np.full(8, -5))
    sg.colored_kv_commit(ctx, cache, i32(table), i32(lens), i32(path), i32(accepted), out, totals=i32(totals))
    commit_oracle(pool, layers, pages << (shift - 1), 1 << (shift - 1), block, heads, dim, table, lens, path, good)
    torch.cuda.synchronize()
    assert out.tolist() == np.where((totals >= 0) & (totals < lens), totals, lens + good).tolist()
    assert torch.equal(d_pool.cpu(), pool)
    assert ctx.device_error() == sg.DEVERR_SEQ
    # all within: no flag, and the same as without totals
    totals = lens + 8
    accepted = np.where(totals > 48, 0, 6)
    totals = np.minimum(totals, 48)
    for kw in (dict(totals=i32(totals)), {}):
        d_pool.copy_(pool)
        sg.colored_kv_commit(ctx, cache, i32(table), i32(lens), i32(path), i32(accepted), out, **kw)
        want = pool.clone()
        commit_oracle(want, layers, pages << (shift - 1), 1 << (shift - 1), block, heads, dim, table, lens, path,
                      accepted)
        torch.cuda.synchronize()
        assert out.tolist() == (lens + accepted).tolist()
        assert torch.equal(d_pool.cpu(), want)
        assert ctx.device_error() == 0


def test_a_request_ends_in_a_step_of_others(ctx):
    """Map, write, attend and commit with the state as it was before the step: the
    request that ends has its old length before and none after, and raises nothing;
    accepted tokens of it do."""
    heads, dim, block, pages = 1, 64, 16, 8
    elems, shift = ko.pages_of(heads, dim, block)
    pool = torch.randn(pages << (shift - 1), generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    d_pool = pool.to(DEV)
    cache = cache_of(d_pool, pages, shift, block, heads, dim, sg.BF16)
    s = State(ctx, 3, 3, pages, block)
    s.lens, _ = s.map([40, 10, 5])
    before = s.lens
    totals, slots = s.map([-1, 3, 0])
    assert totals.tolist() == [0, 13, 5]
    rows = torch.randn(3, 2 * heads, dim, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16)
    q = rows.to(DEV)
    sg.colored_kv_append(ctx, cache, 0, q[:, :1], q[:, 1:], slots)
    out, lse = torch.zeros_like(q), torch.zeros(3, 2, device=DEV)
    work = torch.empty(sg.tree_attention_workspace(cache, 2, 3), dtype=torch.uint8, device=DEV)
    sg.colored_tree_attention(ctx, cache, 0, q, i32([0, 0, 3, 3]), s.table, before, totals, out, work, lse=lse, max_nodes=3,
                              scale=0.125)
    torch.cuda.synchronize()
    assert ctx.device_error() == 0
    at = s.table[1, 0].item() * block + np.arange(13)
    flat, per = d_pool.cpu(), 1 << (shift - 1)
    k, v = (ko.rows(flat, x, per, block, heads, dim, at) for x in (ko.k_index, ko.v_index))
    seen = torch.ones(3, 13, dtype=torch.bool).tril(10)
    o, ls, mass, dots = ko.attend(rows, k, v, seen, 0.125, 0.0)
    ob, lb = ko.attend_bounds(torch.bfloat16, dim, 13, o, ls, mass, dots, 0.0)
    assert bool(((out.cpu().double() - o).abs() <= ob).all()) and bool(((lse.cpu().double() - ls).abs() <= lb).all())
    for first, flag in ((0, 0), (1, sg.DEVERR_SEQ)):
        lens = i32([-1, -1, -1])
        sg.colored_kv_commit(ctx, cache, s.table, before, i32([[0, 1], [0, 1], [0, 0]]), i32([first, 2, 0]), lens,
                             totals=totals)
        assert lens.tolist() == [0, 12, 5] and ctx.device_error() == flag
    assert torch.equal(d_pool.cpu(), flat)
