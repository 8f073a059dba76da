"""The softmax's weights where they meet V, up to 16 rows a segment: held so
closely that the result is the exact one rounded once, and infinite values in
the cache give infinity and no NaN."""
import pytest

import kv_oracle as ko
import paper_2407_13996_amd as sg
from test_gpu_tree_attention import Case

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
FORMS = [(4, 2, 128, [1, 1, 1]), (8, 1, 64, [2, 1, 2]), (2, 1, 96, [8, 3, 1]), (4, 4, 256, [1, 5, 2])]


@pytest.fixture(scope="module")
def ctx():
    c = sg.Context(0)
    yield c
    c.close()


def exact(c):
    out, at = [], 0
    for r, (n_ctx, n) in enumerate(zip(c.lens, c.counts)):
        seen = torch.ones(n, n_ctx + n, dtype=torch.bool)
        seen[:, n_ctx:] = torch.from_numpy(c.seen[r])
        out.append(ko.attend(c.q[at:at + n], c.k[r], c.v[r], seen, c.scale, c.cap)[0])
        at += n
    return torch.cat(out)


@pytest.mark.parametrize("cap", [0.0, 30.0])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv,dim,counts", FORMS)
def test_the_result_is_the_exact_one_rounded_once(ctx, heads, kv, dim, counts, dtype, cap):
    """Rounding o to the type is off by some 0.3 of its unit on average.  A weight
    in two numbers is off by 2^-15 of itself at most (bf16; 2^-21 in f16), sums in fp32
    by (tokens + 64) 2^-24 at most, and errors of many weights mostly
    cancel: less than a tenth of the rounding's, where weights rounded to one
    number of the type are off by as much as o's rounding."""
    c = Case([700, 90, 333], counts, heads, kv, dim, 32, dtype, tree=False, seed=dim, cap=cap)
    out, _ = c.run(ctx)
    want = exact(c)
    rounded = (want.to(dtype).double() - want).square().mean().sqrt()
    off = (out.double() - want).square().mean().sqrt()
    assert float(off) <= 1.1 * float(rounded), float(off / rounded)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv,dim,counts", FORMS)
def test_one_token_gives_its_value(ctx, heads, kv, dim, counts, dtype):
    """A weight of exactly 1: o is v, bit for bit."""
    c = Case([0, 0, 0], [1, 1, 1], heads, kv, dim, 16, dtype, tree=False, seed=1)
    out, _ = c.run(ctx)
    v = torch.cat(c.v).repeat_interleave(heads // kv, 1)
    assert torch.equal(out, v)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv,dim,counts", FORMS)
def test_infinite_values_in_the_cache(ctx, heads, kv, dim, counts, dtype):
    """In steps that every node sees, and in the last one: infinity where there is
    one of one sign, NaN where both or a NaN are, and the other dims as without them."""
    c = Case([100, 40, 64], counts, heads, kv, dim, 16, dtype, tree=False, seed=2)
    clean, lse = c.run(ctx)
    for r, at in ((0, 5), (0, 98), (1, 33), (2, 0)):
        c.v[r][at, :, 0], c.v[r][at, :, 1] = torch.inf, -torch.inf
        c.v[r][at, :, 2] = torch.nan
    c.v[0][50, :, 3], c.v[0][51, :, 3] = torch.inf, -torch.inf
    for r in range(3):
        c.put(r)
    out, again = c.run(ctx)
    assert torch.equal(lse, again)
    assert bool((out[..., 0] == torch.inf).all()) and bool((out[..., 1] == -torch.inf).all())
    assert bool(out[..., 2].isnan().all()) and bool(out[:counts[0], :, 3].isnan().all())
    assert torch.equal(out[counts[0]:, :, 3:], clean[counts[0]:, :, 3:])
    assert torch.equal(out[:, :, 4:], clean[:, :, 4:])
