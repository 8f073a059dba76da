"""Sizes at which the cache's operators take another form: many written
tokens, segments with fewer rows than their form has room for, and caches so
long that one segment's pieces are joined from more ranges than a row's lanes."""
import numpy as np
import pytest

import kv_oracle as ko
import paper_2407_13996_amd as sg
from test_gpu_kv_write import bits, cache_of, slots_of
from test_gpu_tree_attention import Case

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = sg.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("heads,dim,block,n", [(32, 64, 16, 1024), (32, 64, 16, 1025), (32, 96, 32, 2031),
                                               (32, 128, 64, 1500), (32, 256, 16, 1033)])
def test_appends_around_2048_tiles(ctx, heads, dim, block, n):
    rng, gen = np.random.default_rng(n), torch.Generator().manual_seed(n)
    pages = 4 * n // block + 40
    elems, shift = ko.pages_of(heads, dim, block)
    pool = bits(pages << (shift - 1), gen)
    slots = torch.from_numpy(slots_of("runs", n, block, pages, rng).astype(np.int64))
    slots[n // 2:n // 2 + 9] = slots[n // 2:n // 2 + 9].flip(0)   # against the order of memory
    k, v = (bits(n * heads * dim, gen).view(n, heads, dim) for _ in range(2))
    d_pool = pool.to(DEV)
    cache = cache_of(d_pool, pages, shift, block, heads, dim, sg.BF16)
    sg.colored_kv_append(ctx, cache, 0, k.to(DEV).view(torch.bfloat16), v.to(DEV).view(torch.bfloat16),
                         slots.to(DEV))
    on = slots >= 0
    ko.put_rows(pool, ko.k_index, 1 << (shift - 1), block, heads, dim, slots[on], k[on])
    ko.put_rows(pool, ko.v_index, 1 << (shift - 1), block, heads, dim, slots[on], v[on])
    torch.cuda.synchronize()
    assert torch.equal(d_pool.cpu(), pool)
    assert ctx.device_error() == 0


@pytest.mark.parametrize("heads,kv,dim,counts", [
    (8, 2, 128, [60, 1, 33, 5, 28, 64]),      # 4 to 256 rows where 256 have room
    (8, 2, 64, [37, 4, 5, 32, 33, 8]),        # 148 at most
    (6, 2, 96, [43, 5, 6, 10, 11, 42]),       # 129 at most
    (8, 2, 256, [60, 1, 4, 32, 33, 5]),       # wide heads, two blocks of rows
    (4, 1, 128, [32, 1, 3, 4, 5, 13]),        # 128 at most
    (4, 1, 128, [16, 1, 3, 4, 5, 13]),        # 64 at most
])
def test_segments_with_fewer_rows_than_there_is_room_for(ctx, heads, kv, dim, counts):
    for lens in ([700, 64, 65, 0, 1300, 31], [128] * 6):
        c = Case(lens, counts, heads, kv, dim, 32, torch.bfloat16, tree=True, seed=dim + counts[0])
        c.check(*c.run(ctx))
        assert ctx.device_error() == 0


@pytest.mark.parametrize("heads,dim,counts,lens", [(8, 128, [20], [20011]), (2, 256, [2, 1], [20000, 17]),
                                                   (8, 96, [1, 1], [9000, 12001]), (3, 64, [43], [24001])])
def test_segments_in_many_ranges(ctx, heads, dim, counts, lens):
    c = Case(lens, counts, heads, 1, dim, 64, torch.float16, tree=True, seed=dim)
    c.check(*c.run(ctx))
    assert ctx.device_error() == 0
