"""Draft verification over vocabularies below and just at the elements of a 16-byte load (4 of fp32, 8 of bf16 and
fp16), where rows are read element by element, and just above: comparisons, rejections of every token,
draws, rows with nothing and rows with NaN.  Whole numbers, so equal; no random number here lies within
2^-40 of a border but where the sums are exact."""
import pytest

import paper_2407_13996_amd as sg
from test_gpu_draft_verify import TYPES, call, case, compare

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = sg.Context(0)
    yield c
    c.close()


def both(ctx, target, guess, tokens, parents, u, q_start, **kw):
    """With draft rows and without; the counts and tokens of each."""
    out = []
    for host in (guess, None):
        got = call(ctx, target.to(DEV), None if host is None else host.to(DEV), tokens, parents, u, q_start, **kw)
        out.append(compare(ctx, got, target, host, tokens, parents, u, q_start, **kw))
    return out


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", [1, 2, 3, 4, 5, 7, 8, 9])
def test_trees(ctx, vocab, dtype):
    """Chains, broad trees and stars; of most children some are taken and some are not."""
    for i, kind in enumerate(("chain", "tree", "star")):
        args = case([1, 0, 6, 33, 2, 17, 64] * 3, vocab, kind, dtype, 70 + vocab + 10 * i, sharp=1.0)
        taken = [sum(accepted) for accepted, _ in both(ctx, *args)]
        assert sum(taken) > 2 * 18                # more than the roots of the requests that have nodes


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", [1, 2, 3, 5, 7, 8])
def test_every_token_is_rejected(ctx, vocab, dtype):
    """A star with a child for every token, twice, and random numbers that accept next to none: each rejection
    takes its token's weight, and after the last the row itself gives the next token."""
    n = 16
    g = torch.Generator().manual_seed(90 + vocab)
    nodes = 1 + 2 * vocab
    target = torch.softmax(torch.randn(n * nodes, vocab, generator=g), 1).to(TYPES[dtype])
    guess = torch.softmax(torch.randn(n * nodes, vocab, generator=g), 1).to(TYPES[dtype])
    tokens = torch.tensor(([0] + list(range(vocab)) * 2) * n, dtype=torch.int32)
    parents = torch.tensor(([-1] + [0] * 2 * vocab) * n, dtype=torch.int32)
    q_start = torch.arange(0, n * nodes + 1, nodes, dtype=torch.int32)
    u = torch.full((n * nodes,), 1e30)            # above any chance: nothing is accepted
    u[0::nodes] = torch.rand(n, generator=g)
    (drawn, _), (certain, nxt) = both(ctx, target, guess, tokens, parents, u, q_start)
    assert drawn == certain == [1] * n
    # (certain choices: all weights are gone, so the token is the row's own)
    run = torch.cumsum(target[0::nodes].double(), 1)
    assert nxt == (run <= u[0::nodes, None].double() * run[:, -1:]).sum(1).tolist()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", [1, 2, 3, 5, 7, 8])
def test_rows_that_hold_little(ctx, vocab, dtype):
    """Rows of nothing, of one element, of NaN, of negative numbers and infinities, in slices of wider rows that hold
    NaN beside them."""
    inf, nan = float("inf"), float("nan")
    rows = torch.zeros(6 + vocab, vocab)
    rows[0] = nan
    rows[1] = -1.0
    rows[2, ::2], rows[2, 1::2] = nan, 0.25
    rows[3, vocab // 2] = inf
    rows[4] = 1.0 / vocab
    rows[6:] = torch.eye(vocab)                   # (row 5: zeros)
    us = [0.0, 0.375, 0.999, 1.0, nan]
    n = len(rows) * len(us)
    target = rows[:, None].expand(-1, len(us), -1).reshape(n, vocab).repeat_interleave(4, 0).to(TYPES[dtype])
    guess = torch.full((4 * n, vocab), 1.0 / vocab, dtype=TYPES[dtype])
    guess[1::4] = target[1::4]
    tokens = torch.tensor([0, vocab - 1, 0, vocab // 2] * n, dtype=torch.int32)
    parents = torch.tensor([-1, 0, 0, 1] * n, dtype=torch.int32)
    u = torch.tensor(us).repeat(len(rows)).repeat_interleave(4)
    q_start = torch.arange(0, 4 * n + 1, 4, dtype=torch.int32)
    both(ctx, target, guess, tokens, parents, u, q_start)
    wide = torch.full((2, 4 * n, vocab + 5), nan, dtype=TYPES[dtype])
    wide[0, :, 3:3 + vocab], wide[1, :, 1:1 + vocab] = target, guess
    d = wide.to(DEV)
    got = call(ctx, d[0, :, 3:3 + vocab], d[1, :, 1:1 + vocab], tokens, parents, u, q_start, path_stride=3)
    compare(ctx, got, target, guess, tokens, parents, u, q_start, path_stride=3)
