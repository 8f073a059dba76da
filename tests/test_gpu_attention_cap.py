"""Capped scores over the whole range of caps: from caps that all scores reach
to caps so large that they change nothing, where the capped score must be as
exact as one without a cap."""
import pytest

import kv_oracle as ko
import paper_2407_13996_amd as sg
from test_gpu_tree_attention import Case

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ctx():
    c = sg.Context(0)
    yield c
    c.close()


def check(c, out, lse):
    """A capped score is off by what its dot product is (dim + 4 roundings of the
    sum of magnitudes) and 24 more of its own (the cap's factors, e^2y, the
    reciprocal and the series), but never by more than twice the cap.  What
    follows it is rounded as kv_oracle.attend_bounds says."""
    u, e, at = ko.ROUND[c.dtype], 2.0 ** -24, 0
    for r, (ctx_len, n) in enumerate(zip(c.lens, c.counts)):
        t = ctx_len + n
        seen = torch.ones(n, t, dtype=torch.bool)
        seen[:, ctx_len:] = torch.from_numpy(c.seen[r])
        o, ls, mass, dots = ko.attend(c.q[at:at + n], c.k[r], c.v[r], seen, c.scale, c.cap)
        top = 4 * e * torch.where(torch.isinf(ls), 0, ls).abs()
        ds = torch.minimum((c.dim + 28) * e * dots, torch.full_like(dots, 2 * c.cap)) + top
        rest = 2 * ds + (t + 64) * e
        ob = u * o.abs() + (u * (1 + u) + rest[..., None]) * mass + 2.0 ** -24
        got = out[at:at + n].double()
        assert bool(((got - o).abs() <= ob).all()), (r, float(((got - o).abs() - ob).max()))
        g, none = lse[at:at + n].double(), torch.isinf(ls)
        assert torch.equal(g[none], ls[none]), r
        assert bool(((g - ls).abs() <= ds + (t + 64) * e + top)[~none].all()), (r, float((g - ls)[~none].abs().max()))
        at += n


@pytest.mark.parametrize("cap", [1e-3, 0.5, 5.0, 50.0, 300.0, 1e4, 1e6, 1e9, 1e30, 3e38])
@pytest.mark.parametrize("heads,kv,dim,counts,dtype", [
    (4, 2, 128, [1, 1], torch.bfloat16),       # up to 16 rows
    (4, 1, 64, [4, 3], torch.float16),
    (8, 2, 128, [12, 5], torch.bfloat16),      # up to 64
    (8, 1, 96, [16, 2], torch.float16),        # up to 128
    (8, 1, 128, [30, 3], torch.bfloat16),      # up to 256
    (2, 1, 256, [1, 2], torch.float16),        # wide heads
    (4, 1, 256, [33, 4], torch.bfloat16),
])
def test_caps_of_every_size(ctx, heads, kv, dim, counts, dtype, cap):
    for spread in (1.0, 30.0):                 # scores of a few units, and of a hundred
        c = Case([150, 33], counts, heads, kv, dim, 32, dtype, tree=counts[0] > 1, seed=dim + counts[0], cap=cap,
                 spread=spread)
        check(c, *c.run(ctx))
        assert ctx.device_error() == 0


@pytest.mark.parametrize("counts", [[2, 1], [40, 3]])
def test_scales_that_leave_the_caps_range(ctx, counts):
    """scale / cap past fp32's end: every score is the cap or, where the product is 0, 0."""
    c = Case([70, 5], counts, 4, 1, 64, 16, torch.bfloat16, tree=False, seed=3, scale=1e20, cap=1e-20)
    for r, k in enumerate(c.k):
        k[::3] = 0.0
        c.put(r)
    out, lse = c.run(ctx)
    assert not bool(out.isnan().any()) and not bool(lse.isnan().any())
    check(c, out, lse)
    # and a cap of fp32's largest value over a scale that is not 1
    c = Case([70, 5], counts, 4, 1, 64, 16, torch.float16, tree=False, seed=3, scale=0.01,
             cap=float(torch.finfo(torch.float32).max))
    check(c, *c.run(ctx))
