"""Verification of drafted trees against the rule on the host: whole numbers, so equal, where a
random number does not lie within 2^-40 of a border (the probabilities are such that none does, or the
borders are exact)."""
import numpy as np
import pytest

import paper_2407_13996_amd as sg
import verify_oracle as vo

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def ctx():
    c = sg.Context(0)
    yield c
    c.close()


def trees(counts, vocab, kind, g):
    """Tokens and parents of random trees: chains, broad trees, stars."""
    parents, tokens = [], []
    for n in counts:
        for i in range(n):
            r = float(torch.rand((), generator=g))
            parents.append(-1 if i == 0 else i - 1 if kind == "chain" else 0 if kind == "star" else
                           max(0, i - 1 - int(r * 6)))
            tokens.append(int(torch.randint(0, vocab, (), generator=g)))
    return torch.tensor(tokens, dtype=torch.int32), torch.tensor(parents, dtype=torch.int32)


def case(counts, vocab, kind, dtype, seed, sharp=4.0):
    g = torch.Generator().manual_seed(seed)
    n = sum(counts)
    x = sharp * torch.randn(n, vocab, generator=g)
    target = torch.softmax(x, 1)
    guess = torch.softmax(x + torch.randn(n, vocab, generator=g), 1)
    tokens, parents = trees(counts, vocab, kind, g)
    # most tokens are likely ones under their parent
    start = 0
    for c in counts:
        for i in range(1, c):
            if torch.rand((), generator=g) < 0.8:
                row = guess[start + max(int(parents[start + i]), 0)]
                tokens[start + i] = int(row.topk(min(4, vocab)).indices[int(torch.randint(0, min(4, vocab), (), generator=g))])
        start += c
    q_start = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32)
    return target.to(TYPES[dtype]), guess.to(TYPES[dtype]), tokens, parents, torch.rand(n, generator=g), q_start


def call(ctx, target, draft, tokens, parents, u, q_start, path_stride=None, max_nodes=256, stream=None, **lens):
    n = q_start.numel() - 1
    path = torch.full((n, path_stride or 256), 77, dtype=torch.int32, device=DEV)
    accepted, nxt = (torch.full((n,), 77, dtype=torch.int32, device=DEV) for _ in range(2))
    sg.colored_draft_verify(ctx, target, tokens.to(DEV), parents.to(DEV), u.to(DEV), q_start.to(DEV), path, accepted,
                            nxt, draft=draft, max_nodes=max_nodes, stream=stream,
                            **{k: v.to(DEV) for k, v in lens.items()})
    return path, accepted, nxt


def compare(ctx, got, target, draft, tokens, parents, u, q_start, path_stride=None, max_nodes=256, **lens):
    f = lambda t: None if t is None else t.cpu().double().numpy()  # noqa: E731
    paths, accepted, nxt, flag = vo.verify(f(target), f(draft), tokens.numpy(), parents.numpy(), u.double().numpy(),
                                           q_start.numpy(), path_stride or 256, max_nodes,
                                           **{k: v.numpy() for k, v in lens.items()})
    torch.cuda.synchronize()
    assert got[1].tolist() == accepted
    assert got[0].tolist() == paths
    assert got[2].tolist() == nxt
    assert ctx.device_error() == (sg.DEVERR_SEQ if flag else 0)
    return accepted, nxt


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("counts,vocab,kind,dtype", [
    ([1], 1, "chain", "f32"), ([5], 33, "chain", "f32"), ([1, 0, 3, 17], 257, "tree", "bf16"),
    ([8] * 9, 1023, "chain", "f16"), ([60, 1, 64, 65], 1025, "tree", "f32"), ([256], 2049, "tree", "f32"),
    ([256], 500, "star", "f32"), ([7, 9], 50257, "tree", "bf16"), ([4, 5, 6], 131072, "chain", "f32"),
    ([3], 600011, "tree", "f16"), ([2] * 300, 64, "chain", "f32"), ([12] * 40, 4097, "tree", "f32")])
def test_trees(ctx, counts, vocab, kind, dtype, drawn):
    target, guess, tokens, parents, u, q_start = case(counts, vocab, kind, dtype, vocab + len(counts))
    t, d = target.to(DEV), guess.to(DEV) if drawn else None
    got = call(ctx, t, d, tokens, parents, u, q_start)
    compare(ctx, got, target, guess if drawn else None, tokens, parents, u, q_start)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_anywhere(ctx, dtype):
    """Rows that are slices of wider ones, at odd elements; draft rows apart from the target's."""
    target, guess, tokens, parents, u, q_start = case([6, 1, 9], 1001, "tree", dtype, 3)
    wide_t = torch.full((16, 1777), float("nan"), dtype=target.dtype)
    wide_d = torch.full((16, 1235), float("nan"), dtype=target.dtype)
    wide_t[:, 5:1006], wide_d[:, 1:1002] = target, guess
    args = tokens, parents, u, q_start
    got = call(ctx, wide_t.to(DEV)[:, 5:1006], wide_d.to(DEV)[:, 1:1002], *args)
    compare(ctx, got, target, guess, *args)
    got = call(ctx, wide_t.to(DEV)[:, 5:1006], None, *args)
    compare(ctx, got, target, None, *args)


def test_borders(ctx):
    """Probabilities that are multiples of 2^-6: all sums are exact, and a random number on a border
    belongs to the next token; a chance equal to the random number is not enough."""
    vocab = 64
    target = torch.full((64 * 2, vocab), 2.0 ** -6)
    tokens = torch.tensor([0, 9] * 64, dtype=torch.int32)
    parents = torch.tensor([-1, 0] * 64, dtype=torch.int32)
    u = torch.zeros(128)
    u[0::2] = torch.arange(64) / 64.0         # the draw: v / 64 gives v
    u[1::2] = 2.0 ** -6                       # equal to the chance: rejected
    q_start = torch.arange(0, 129, 2, dtype=torch.int32)
    got = call(ctx, target.to(DEV), None, tokens, parents, u, q_start)
    accepted, nxt = compare(ctx, got, target, None, tokens, parents, u, q_start)
    assert accepted == [1] * 64 and 9 not in nxt and nxt[0] == 0
    u[1::2] = 2.0 ** -6 - 2.0 ** -30          # just below: accepted, and the child's row gives v
    got = call(ctx, target.to(DEV), None, tokens, parents, u, q_start)
    accepted, nxt = compare(ctx, got, target, None, tokens, parents, u, q_start)
    assert accepted == [2] * 64 and nxt == list(range(64))


def test_odd_probabilities_and_random_numbers(ctx):
    """Zeros, rows of nothing, NaN, infinities, negative numbers; random numbers outside [0, 1)."""
    inf, nan = float("inf"), float("nan")
    rows = [[0, 0, 0, 0, 0], [0, 1, 0, 0, 0], [nan, 0.5, -1, 0.5, nan], [0, inf, 0, 1, 0], [-0.0, 0, 0, 0, 1e-45],
            [nan] * 5, [-inf, -1, nan, 0, -0.0], [0.2] * 5, [inf, inf, 0, 0, 0], [1, 1, 1, 1, 1]]
    us = [0.0, 0.25, 0.999999, 1.0, 2.0, -1.0, nan, inf]
    n = len(rows) * len(us)
    for drawn in (False, True):
        target = torch.tensor(rows)[:, None].expand(len(rows), len(us), 5).reshape(n, 5).repeat_interleave(3, 0)
        guess = torch.tensor([0.0, 0.5, 0.0, 0.5, 0.0]).expand(3 * n, 5).contiguous()
        tokens = torch.tensor([0, 1, 3] * n, dtype=torch.int32)
        parents = torch.tensor([-1, 0, 0] * n, dtype=torch.int32)
        u = torch.tensor(us).repeat(len(rows)).repeat_interleave(3)
        q_start = torch.arange(0, 3 * n + 1, 3, dtype=torch.int32)
        d = guess if drawn else None
        got = call(ctx, target.to(DEV), None if d is None else d.to(DEV), tokens, parents, u, q_start)
        compare(ctx, got, target, d, tokens, parents, u, q_start)


def test_nothing_left(ctx):
    """A rejected certain choice that was all there was: the row itself gives the token. The same
    for a draft that covers the target everywhere."""
    target = torch.zeros(2, 7)
    target[:, 4] = 1 - 2.0 ** -24
    tokens, parents = torch.tensor([0, 4], dtype=torch.int32), torch.tensor([-1, 0], dtype=torch.int32)
    u, q_start = torch.tensor([0.3, 1 - 2.0 ** -24]), torch.tensor([0, 2], dtype=torch.int32)
    for draft in (None, target * (1 + 2.0 ** -20)):
        got = call(ctx, target.to(DEV), None if draft is None else draft.to(DEV), tokens, parents, u, q_start)
        compare(ctx, got, target, draft, tokens, parents, u, q_start)
        assert got[2].tolist() == [4] and got[1].tolist() == [1]


def test_requests_that_are_not_served_and_arrays_out_of_range(ctx):
    target, guess, tokens, parents, u, q_start = case([4, 6, 2, 5], 300, "chain", "f32", 9)
    t, d = target.to(DEV), guess.to(DEV)
    lens = torch.tensor([10, 0, 7, 3], dtype=torch.int32)
    totals = torch.tensor([14, 0, 9, 7], dtype=torch.int32)     # 1 and 3 were not served
    got = call(ctx, t, d, tokens, parents, u, q_start, lens=lens, totals=totals)
    accepted, nxt = compare(ctx, got, target, guess, tokens, parents, u, q_start, lens=lens, totals=totals)
    assert accepted[1] == accepted[3] == 0 and nxt[1] == nxt[3] == -1
    # tokens and parents that are none
    bad, strange = tokens.clone(), parents.clone()
    bad[1], bad[5], strange[7], strange[13] = 300, -1, 9, -5
    got = call(ctx, t, d, bad, strange, u, q_start)
    compare(ctx, got, target, guess, bad, strange, u, q_start)
    # short paths, more nodes than said, starts out of order and past the nodes
    for kw in (dict(path_stride=1), dict(path_stride=2), dict(max_nodes=3), dict(max_nodes=1)):
        got = call(ctx, t, d, tokens, parents, u, q_start, **kw)
        compare(ctx, got, target, guess, tokens, parents, u, q_start, **kw)
    for starts in ([0, 4, 3, 12, 17], [0, 4, 10, 12, 18], [5, 4, 3, 2, 1]):
        s = torch.tensor(starts, dtype=torch.int32)
        got = call(ctx, t, d, tokens, parents, u, s)
        compare(ctx, got, target, guess, tokens, parents, u, s)


def test_no_nodes_at_all(ctx):
    empty = torch.zeros(0, 9, device=DEV)
    got = call(ctx, empty, None, torch.zeros(0, dtype=torch.int32), torch.zeros(0, dtype=torch.int32), torch.zeros(0),
               torch.zeros(4, dtype=torch.int32), path_stride=3)
    torch.cuda.synchronize()
    assert got[0].tolist() == [[-1] * 3] * 3 and got[1].tolist() == [0] * 3 and got[2].tolist() == [-1] * 3
    assert ctx.device_error() == 0


def test_any_cus_and_streams(ctx):
    target, guess, tokens, parents, u, q_start = case([9] * 50, 5000, "tree", "f32", 11)
    t, d = target.to(DEV), guess.to(DEV)
    s = torch.cuda.Stream()
    for cus in (None, range(32), [3, 70, 71], [255]):
        s.wait_stream(torch.cuda.current_stream())
        sg.set_cu_mask(ctx, s, cus)
        with torch.cuda.stream(s):
            got = call(ctx, t, d, tokens, parents, u, q_start, stream=s)
        s.synchronize()
        compare(ctx, got, target, guess, tokens, parents, u, q_start)
    sg.stream_release(ctx, s)


def test_captured_and_replayed(ctx):
    counts = [7, 3, 9]
    target, guess, tokens, parents, u, q_start = case(counts, 2000, "tree", "f32", 12)
    bufs = [x.to(DEV) for x in (target, guess, tokens, parents, u, q_start)]
    path = torch.zeros(3, 16, dtype=torch.int32, device=DEV)
    accepted, nxt = (torch.zeros(3, dtype=torch.int32, device=DEV) for _ in range(2))

    def go():
        t, d, k, p, x, s = bufs
        sg.colored_draft_verify(ctx, t, k, p, x, s, path, accepted, nxt, draft=d)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        go()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        go()
    for seed in range(4):
        new = case(counts, 2000, "tree", "f32", 40 + seed)
        for b, x in zip(bufs, new):
            b.copy_(x)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        compare(ctx, (path, accepted, nxt), *new, path_stride=16)
        go()
        compare(ctx, (path, accepted, nxt), *new, path_stride=16)
    sg.stream_release(ctx, s)


def test_rows_past_4_gib(ctx):
    """The second request's rows begin past 2^32 bytes."""
    vocab, stride = 1000, 1 << 29
    target, guess, tokens, parents, u, q_start = case([2, 3], vocab, "chain", "f32", 13)
    pool = torch.zeros(4 * stride + vocab, device=DEV)
    rows = pool.as_strided((5, vocab), (stride, 1))
    rows.copy_(target)
    got = call(ctx, rows, guess.to(DEV), tokens, parents, u, q_start)
    compare(ctx, got, target, guess, tokens, parents, u, q_start)


def test_the_tokens_are_distributed_as_the_targets(ctx):
    """Two children drawn from the draft, then the draw: over 64 rounds of 4096 requests each token
    comes up as often as its probability says, within five standard deviations."""
    g = torch.Generator().manual_seed(14)
    vocab, n = 12, 4096
    p, q = torch.softmax(torch.randn(vocab, generator=g), 0), torch.softmax(torch.randn(vocab, generator=g), 0)
    target, guess = p.expand(3 * n, vocab).contiguous().to(DEV), q.expand(3 * n, vocab).contiguous().to(DEV)
    parents = torch.tensor([-1, 0, 0] * n, dtype=torch.int32)
    q_start = torch.arange(0, 3 * n + 1, 3, dtype=torch.int32)
    seen = torch.zeros(vocab, dtype=torch.int64)
    for _ in range(64):
        tokens = torch.multinomial(q, 3 * n, replacement=True, generator=g).to(torch.int32)
        u = torch.rand(3 * n, generator=g)
        path, accepted, nxt = (t.cpu() for t in call(ctx, target, guess, tokens, parents, u, q_start, path_stride=2))
        first = torch.where(accepted == 2, tokens.view(n, 3).gather(1, path[:, 1:].clamp(min=0).long())[:, 0], nxt)
        seen += torch.bincount(first.long(), minlength=vocab)
    total = 64 * n
    sigma = torch.sqrt(total * p.double() * (1 - p.double()))
    assert bool(((seen - total * p.double()).abs() <= 5 * sigma).all())


@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_shared_by_workgroups(ctx, dtype):
    """Few requests over long rows, on CU masks that give each from sixteen workgroups to one, a graph
    of two calls in a row with other inputs every replay, and launches between the replays."""
    counts, vocab = [5, 0, 9], 270001
    arrays = [case(counts, vocab, kind, dtype, 30 + i) for i, kind in enumerate(("chain", "tree", "star"))]
    s = torch.cuda.Stream()
    for cus in (None, range(64), range(12), [40, 41, 7], [17]):
        sg.set_cu_mask(ctx, s, cus)
        for args in arrays:
            target, guess, *rest = args
            t, d = target.to(DEV), guess.to(DEV)
            s.wait_stream(torch.cuda.current_stream())
            for draft, host in ((d, guess), (None, None)):
                with torch.cuda.stream(s):
                    got = call(ctx, t, draft, *rest)
                s.synchronize()
                compare(ctx, got, target, host, *rest)
    sg.set_cu_mask(ctx, s, None)
    bufs = [x.to(DEV) for x in arrays[0]]
    outs = [[torch.zeros(3, 16, dtype=torch.int32, device=DEV)] +
            [torch.zeros(3, dtype=torch.int32, device=DEV) for _ in range(2)] for _ in range(2)]

    def go(out, drawn):
        t, d, k, p, u, q = bufs
        sg.colored_draft_verify(ctx, t, k, p, u, q, *out, draft=d if drawn else None)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        go(outs[0], True)
        go(outs[1], False)
    for args in arrays + arrays[:1]:
        for b, x in zip(bufs, args):
            b.copy_(x)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        compare(ctx, outs[0], *args, path_stride=16)
        compare(ctx, outs[1], args[0], None, *args[2:], path_stride=16)
        with torch.cuda.stream(s):
            go(outs[0], False)
        s.synchronize()
        compare(ctx, outs[0], args[0], None, *args[2:], path_stride=16)
    sg.stream_release(ctx, s)


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_odd_probabilities_among_many(ctx, dtype, drawn):
    """One element in a thousand is NaN, infinite, negative, -0 or the smallest there is, so that some
    runs of a row hold such elements and others none; an infinity counts as the largest fp32 and
    leaves the draw to itself, so that most rows have none."""
    target, guess, tokens, parents, u, q_start = case([7, 5, 30, 1, 12, 9], 20011, "tree", dtype, 60)
    g = torch.Generator().manual_seed(61)
    least = torch.tensor([1], dtype=torch.int32 if dtype == "f32" else torch.int16).view(TYPES[dtype])[0].item()
    for t in (target, guess):
        n = t.numel() // 1000
        at = torch.randperm(t.numel(), generator=g)[:n]
        odd = torch.tensor([float("nan"), -0.5, -0.0, least, float("-inf"), -float("nan")], dtype=t.dtype)
        t.view(-1)[at] = odd[torch.randint(0, len(odd), (n,), generator=g)]
    target[3, 15000] = target[40, 3] = guess[20, 777] = float("inf")
    got = call(ctx, target.to(DEV), guess.to(DEV) if drawn else None, tokens, parents, u, q_start)
    compare(ctx, got, target, guess if drawn else None, tokens, parents, u, q_start)
