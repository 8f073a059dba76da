"""The cache's calls on block tables that are slices of wider ones: a request
has the blocks of its row of the slice and no more, and what lies beside the
slice is neither written nor taken for pages."""
import numpy as np
import pytest

import kv_oracle as ko
import paper_2407_13996_amd as sg
from test_gpu_kv_write import bits, cache_of, commit_oracle
from test_gpu_tree_attention import Case

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
MARK = 7777


@pytest.fixture(scope="module")
def ctx():
    c = sg.Context(0)
    yield c
    c.close()


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a).astype(np.int32))).to(DEV)


def inside(rows, before=2, after=3):
    """``rows`` as a slice of a wider table of marks, with rows of marks around it."""
    n, width = np.shape(rows)
    big = torch.full((n + 2, before + width + after), MARK, dtype=torch.int32, device=DEV)
    view = big[1:1 + n, before:before + width]
    view.copy_(i32(rows))
    return big, view


def beside(big, view, before=2):
    """Marks beside the slice, all of them if nothing was written there."""
    rest = big.clone()
    rest[1:1 + view.shape[0], before:before + view.shape[1]] = MARK
    return bool((rest == MARK).all())


@pytest.mark.parametrize("requests", [1, 3, 300])
def test_requests_get_no_more_blocks_than_the_slice_has(ctx, requests):
    """Every third request asks for one token more than its row holds, the others for all of it."""
    block, width, pages = 16, 6, 6 * requests
    rng = np.random.default_rng(requests)
    new = np.where(np.arange(requests) % 3 == 0, block * width + 1, block * width)
    tokens, ring = int(new.sum()), rng.permutation(pages).astype(np.int32)
    table = np.full((requests, width), -1, np.int32)
    big, view = inside(table)
    held = np.zeros(requests, int)
    d_ring, pos = i32(ring), torch.tensor([0, pages], dtype=torch.int64, device=DEV)
    out = {"ring_pos": torch.zeros_like(pos), "held": i32(held), "lens": i32(held),
           "q_start": i32(np.zeros(requests + 1)), "slots": torch.zeros(tokens, dtype=torch.int64, device=DEV),
           "request": i32(np.zeros(tokens)), "position": i32(np.zeros(tokens))}
    sg.colored_kv_map(ctx, block, d_ring, pos, i32(held), i32(held), i32(new), view, out["ring_pos"], out["held"],
                      out["lens"], out["q_start"], out["slots"], out["request"], out["position"])
    torch.cuda.synchronize()
    want = ko.kv_map(block, ring, [0, pages], held, held, new, table, tokens)
    assert want.pop("flag") and ctx.device_error() == sg.DEVERR_SEQ
    for k, w in want.items():
        assert np.array_equal(out[k].cpu().numpy(), np.asarray(w)), k
    assert np.array_equal(view.cpu().numpy(), table)
    assert beside(big, view)


@pytest.mark.parametrize("requests", [1, 2])
def test_paths_are_cut_at_the_slices_end(ctx, requests):
    """A path that leaves the row, over pages that the entries beside it would name."""
    heads, dim, block, pages = 2, 64, 16, 12
    elems, shift = ko.pages_of(heads, dim, block)
    pool = bits(pages << (shift - 1), torch.Generator().manual_seed(2))
    table = np.arange(2 * requests).reshape(requests, 2)
    big, view = inside(table)
    big[big == MARK] = 9                                # a page of the pool
    lens, accepted = np.full(requests, 28), np.full(requests, 3)
    path = np.tile([1, 3, 4], (requests, 1))            # 28 + 4 is the first token past two blocks
    d_pool, out = pool.to(DEV), i32(np.zeros(requests))
    sg.colored_kv_commit(ctx, cache_of(d_pool, pages, shift, block, heads, dim, sg.BF16), view, i32(lens), i32(path),
                         i32(accepted), out)
    commit_oracle(pool, 1, 0, 1 << (shift - 1), block, heads, dim, table, lens, path, np.full(requests, 2))
    torch.cuda.synchronize()
    assert out.cpu().tolist() == [30] * requests
    assert torch.equal(d_pool.cpu(), pool)
    assert ctx.device_error() == sg.DEVERR_SEQ


@pytest.mark.parametrize("nodes,heads,dim", [(1, 4, 64), (9, 8, 128)])
def test_attention_over_a_slice(ctx, nodes, heads, dim):
    """As over a table of its own; and a cache said to be longer than its row is read to the row's end."""
    c = Case([40, 64, 7], [nodes] * 3, heads, 2, dim, 16, torch.bfloat16, tree=nodes > 1, seed=5)
    width = -(-max(c.totals) // 16)
    c.table = c.table[:, :width]
    want, lse = c.run(ctx)
    c.check(want, lse)
    assert ctx.device_error() == 0
    pool, q, work, wide = c.keep
    big, view = inside(c.table)
    big[big == MARK] = 0                                # a page of the pool
    cache = sg.kv_cache(pool, c.pages, c.shift, 16, 2, dim, sg.BF16)
    got, other = torch.zeros_like(want, device=DEV), torch.zeros_like(lse, device=DEV)

    def call(lens, totals):
        sg.colored_tree_attention(ctx, cache, 0, q, i32(np.arange(4) * nodes), view, i32(lens), i32(totals), got, work,
                                  lse=other, mask=None if c.mask is None else c.mask.to(DEV), max_nodes=nodes,
                                  scale=c.scale)
        torch.cuda.synchronize()
        return ctx.device_error()

    assert call(c.lens, c.totals) == 0
    assert torch.equal(got.cpu(), want) and torch.equal(other.cpu(), lse)
    cap = width * 16
    short = [cap - nodes] * 3
    assert call(short, [cap, cap, cap]) & ~sg.DEVERR_PT_RANGE == 0
    clamped, other_lse = got.clone(), other.clone()
    assert call(short, [cap, cap + 1, 2 ** 31 - 1]) & ~sg.DEVERR_PT_RANGE == sg.DEVERR_SEQ
    assert torch.equal(got.view(torch.int16), clamped.view(torch.int16))
    assert torch.equal(other.view(torch.int32), other_lse.view(torch.int32))
