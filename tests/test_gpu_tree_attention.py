"""Attention of drafted tokens over the paged cache, against 64-bit loops on
the host with bounds derived from the kernel's roundings (kv_oracle)."""
import numpy as np
import pytest

import kv_oracle as ko
import paper_2407_13996_amd as sg

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
CODE = {torch.bfloat16: sg.BF16, torch.float16: sg.F16}


@pytest.fixture(scope="module")
def ctx():
    c = sg.Context(0)
    yield c
    c.close()


def tree_masks(counts, words, rng, empty=True):
    """Bits of random trees' ancestors; some nodes see nothing, some only later ones."""
    total = sum(counts)
    seen = [np.zeros((c, c), bool) for c in counts]
    for m in seen:
        for i in range(len(m)):
            if i:
                m[i] = m[rng.integers(0, i)]
            m[i, i] = True
        if empty and len(m) > 2:
            m[len(m) // 2] = False
            m[len(m) - 2] = rng.random(len(m)) < 0.5
    bits = np.zeros((total, words), np.uint64)
    at = 0
    for m in seen:
        for i in range(len(m)):
            for j in np.nonzero(m[i])[0]:
                bits[at, j // 64] |= np.uint64(1) << np.uint64(j % 64)
            at += 1
    return seen, torch.from_numpy(bits.view(np.int64))


class Case:
    """Requests with ``lens`` cached and ``counts`` drafted tokens; the rest of
    the pool (and of the last blocks) holds NaN."""

    def __init__(self, lens, counts, heads, kv, dim, block, dtype, tree, seed=0, scale=None, cap=0.0, spread=1.0):
        self.lens, self.counts, self.heads, self.kv, self.dim, self.block = lens, counts, heads, kv, dim, block
        self.dtype, self.cap = dtype, cap
        self.scale = dim ** -0.5 if scale is None else scale
        rng, gen = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
        self.totals = [a + b for a, b in zip(lens, counts)]
        n, used = len(lens), [-(-t // block) for t in self.totals]
        self.elems, self.shift = ko.pages_of(kv, dim, block)
        self.pages, width = sum(used) + 2, max(max(used), 1) + 1
        perm, at = rng.permutation(self.pages), 0
        self.table = np.full((n, width), -1, np.int64)
        for r, u in enumerate(used):
            self.table[r, :u] = perm[at:at + u]
            at += u
        self.per = 1 << (self.shift - 1)
        self.pool = torch.full((self.pages * self.per,), torch.nan, dtype=dtype)
        self.k, self.v = [], []
        for r, t in enumerate(self.totals):
            k = (torch.randn(t, kv, dim, generator=gen) * spread).to(dtype)
            v = torch.randn(t, kv, dim, generator=gen).to(dtype)
            self.k.append(k)
            self.v.append(v)
            self.put(r)
        tokens = sum(counts)
        self.proj = torch.randn(tokens, heads + 2, dim, generator=gen).to(dtype)
        self.q = self.proj[:, 1:1 + heads]
        self.words = -(-max(max(counts), 1) // 64)
        if tree:
            self.seen, self.mask = tree_masks(counts, self.words, rng)
        else:
            self.seen, self.mask = [np.tril(np.ones((c, c), bool)) for c in counts], None

    def slots(self, r):
        p = np.arange(self.totals[r])
        return torch.from_numpy(self.table[r, p // self.block] * self.block + p % self.block)

    def put(self, r):
        if self.totals[r]:
            for index, x in ((ko.k_index, self.k[r]), (ko.v_index, self.v[r])):
                ko.put_rows(self.pool, index, self.per, self.block, self.kv, self.dim, self.slots(r), x)

    def run(self, ctx, lse=True, stream=None, totals=None, table=None, pool=None):
        i32 = lambda a: torch.from_numpy(np.asarray(a).astype(np.int32)).to(DEV)  # noqa: E731
        pool = self.pool.to(DEV) if pool is None else pool
        cache = sg.kv_cache(pool, self.pages, self.shift, self.block, self.kv, self.dim, CODE[self.dtype])
        q = self.proj.to(DEV)[:, 1:1 + self.heads]
        most = max(max(self.counts), 1)
        work = torch.empty(sg.tree_attention_workspace(cache, self.heads, most), dtype=torch.uint8, device=DEV)
        work.fill_(0xFF)  # NaN
        # every row of a wider buffer, to see that nothing beside it is written
        wide = torch.full((sum(self.counts), self.heads + 3, self.dim), 7.0, dtype=self.dtype, device=DEV)
        out = wide[:, 2:2 + self.heads]
        self.d_lse = torch.full((sum(self.counts), self.heads), 7.0, device=DEV) if lse else None
        self.keep = (pool, q, work, wide)
        args = (cache, 0, q, i32(np.concatenate([[0], np.cumsum(self.counts)])),
                i32(self.table if table is None else table), i32(self.lens),
                i32(self.totals if totals is None else totals), out, work)
        kw = dict(lse=self.d_lse, mask=None if self.mask is None else self.mask.to(DEV), max_nodes=most,
                  scale=self.scale, softcap=self.cap, stream=stream)
        self.call = lambda: sg.colored_tree_attention(ctx, *args, **kw)
        self.call()
        torch.cuda.synchronize()
        assert bool((wide[:, :2] == 7).all()) and bool((wide[:, 2 + self.heads:] == 7).all())
        self.out = out
        return out.cpu(), None if not lse else self.d_lse.cpu()

    def check(self, out, lse, drafted=None):
        at = 0
        for r, (c, n) in enumerate(zip(self.lens, self.counts)):
            d = n if drafted is None else drafted[r]
            seen = torch.ones(n, c + d, dtype=torch.bool)
            seen[:, c:] = torch.from_numpy(self.seen[r])[:, :d]
            o, ls, mass, dots = ko.attend(self.q[at:at + n], self.k[r][:c + d], self.v[r][:c + d], seen, self.scale,
                                          self.cap)
            ob, lb = ko.attend_bounds(self.dtype, self.dim, c + d, o, ls, mass, dots, self.cap)
            got = out[at:at + n].double()
            assert bool(((got - o).abs() <= ob).all()), (r, float(((got - o).abs() - ob).max()))
            if lse is not None:
                g, none = lse[at:at + n].double(), torch.isinf(ls)
                assert torch.equal(g[none], ls[none]), r
                assert bool(((g - ls).abs() <= lb)[~none].all()), (r, float(((g - ls).abs() - lb)[~none].max()))
            at += n


EDGES = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 500]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,kv,dim,block", [(4, 1, 64, 16), (7, 7, 96, 32), (8, 2, 128, 64), (16, 2, 128, 16),
                                                (6, 2, 256, 128), (15, 5, 64, 1024)])
def test_single_tokens_over_ragged_caches(ctx, heads, kv, dim, block, dtype):
    c = Case(EDGES, [1] * len(EDGES), heads, kv, dim, block, dtype, tree=False, seed=dim)
    c.check(*c.run(ctx))
    assert ctx.device_error() == 0


@pytest.mark.parametrize("heads,kv,dim,block,lens,counts,dtype,cap", [
    (4, 2, 128, 64, [0, 100, 31, 0, 64], [5, 8, 1, 1, 7], torch.bfloat16, 0.0),      # up to 16 rows
    (8, 2, 128, 32, [0, 700, 3], [8, 5, 7], torch.float16, 30.0),                     # 32 rows
    (8, 2, 64, 16, [40, 0, 95], [13, 16, 1], torch.bfloat16, 0.0),                     # 64 rows
    (6, 2, 96, 16, [1, 230], [20, 17], torch.float16, 0.0),                            # 64 rows, a group of three
    (16, 2, 128, 64, [300, 5], [16, 11], torch.bfloat16, 50.0),                        # 128 rows
    (8, 1, 128, 16, [33, 90], [30, 2], torch.float16, 0.0),                            # 256 rows
    (8, 1, 64, 32, [10, 257, 0], [64, 1, 65], torch.bfloat16, 0.0),                    # more than a block of rows
    (2, 1, 128, 64, [130], [256], torch.bfloat16, 0.0),                                # the largest draft
    (2, 1, 256, 16, [70, 0], [16, 9], torch.bfloat16, 20.0),                           # wide heads, 32 rows
    (4, 1, 256, 64, [200, 31], [16, 3], torch.float16, 0.0),                           # 64 rows
    (8, 2, 256, 32, [64, 7], [33, 40], torch.bfloat16, 0.0),                           # more than 128 rows
])
def test_trees_and_chains(ctx, heads, kv, dim, block, lens, counts, dtype, cap):
    for tree in (True, False):
        c = Case(lens, counts, heads, kv, dim, block, dtype, tree, seed=sum(counts), cap=cap)
        c.check(*c.run(ctx))
        assert ctx.device_error() == 0


@pytest.mark.parametrize("dtype,counts", [(torch.bfloat16, [1]), (torch.float16, [3, 1]), (torch.bfloat16, [20, 9])])
def test_long_caches_are_split_and_joined(ctx, dtype, counts):
    """Far more steps than a wavefront takes alone: pieces of a segment in many ranges."""
    lens = [9000, 2500][:len(counts)]
    c = Case(lens, counts, 4, 1, 64, 16, dtype, tree=len(counts) > 1, seed=3)
    out, lse = c.run(ctx)
    c.check(out, lse)


def test_large_and_small_scores(ctx):
    """Scores of hundreds: one token takes all the weight; and nearly equal ones."""
    for spread, scale in ((40.0, 1.0), (1e-3, None)):
        c = Case([200, 33], [3, 2], 4, 2, 64, 16, torch.bfloat16, tree=False, seed=9, spread=spread, scale=scale)
        c.check(*c.run(ctx))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_what_is_not_seen_does_not_reach_a_row(ctx, dtype):
    """Drafted tokens with infinite and NaN keys and values: nodes that do not
    see them are as if they were not there, nodes that do get what the formula gives."""
    for heads, dim, counts in ((2, 64, [9, 4]), (8, 128, [20, 3]), (8, 64, [30, 2]), (2, 256, [9, 4])):
        c = Case([45, 0], counts, heads, 1, dim, 16, dtype, tree=True, seed=4)
        for m in c.seen:  # nodes see themselves and the first node only
            m[:] = np.eye(len(m), dtype=bool)
            m[:, 0] = True
        bits = np.zeros((sum(counts), 1), np.uint64)
        at = 0
        for m in c.seen:
            for i in range(len(m)):
                bits[at, 0] = np.uint64(1) | np.uint64(1) << np.uint64(i)
                at += 1
        c.mask = torch.from_numpy(bits.view(np.int64))
        clean_out, clean_lse = c.run(ctx)
        k, v = c.k[0], c.v[0]
        k[45 + 2] = torch.nan                     # node 2 sees a NaN score
        v[45 + 3, 0, 0], v[45 + 3, 0, 1] = torch.inf, -torch.inf
        v[45 + 4, 0, dim - 1] = torch.nan
        k[45 + 5], v[45 + 5] = 0.0, torch.inf
        v[45 + 6, 0, :] = -torch.inf
        c.put(0)
        out, lse = c.run(ctx)
        clean = torch.ones(sum(counts), dtype=torch.bool)
        clean[[2, 3, 4, 5, 6]] = False
        assert torch.equal(out[clean], clean_out[clean]) and torch.equal(lse[clean], clean_lse[clean])
        assert bool(out[2].isnan().all()) and bool(lse[2].isnan().all())
        assert bool((out[3, :, 0] == torch.inf).all()) and bool((out[3, :, 1] == -torch.inf).all())
        assert torch.equal(out[3, :, 2:], clean_out[3, :, 2:])
        assert bool(out[4, :, dim - 1].isnan().all()) and torch.equal(out[4, :, :-1], clean_out[4, :, :-1])
        assert bool((out[5] == torch.inf).all()) and bool((out[6] == -torch.inf).all())


def test_drafted_tokens_without_pages(ctx):
    """A request that got no pages for its draft: its nodes see what is cached, or nothing."""
    c = Case([50, 0, 33], [3, 4, 2], 4, 2, 64, 16, torch.bfloat16, tree=False, seed=6)
    out, lse = c.run(ctx, totals=[50, 0, 35])
    c.check(out, lse, drafted=[0, 0, 2])
    assert bool((out[3:7] == 0).all()) and bool((lse[3:7] == -torch.inf).all())


def test_without_lse_and_on_a_mask_of_single_cus(ctx):
    """The same bits on all CUs, on some XCDs, on scattered CUs, with pieces of
    any length a workgroup, on a stream of its own, and when repeated."""
    c = Case([900, 0, 77, 5000], [6, 1, 12, 3], 8, 2, 128, 32, torch.bfloat16, tree=True, seed=8)
    want, lse = c.run(ctx)
    c.check(want, lse)
    assert torch.equal(c.run(ctx, lse=False)[0], want)
    for cus in (range(32), range(64, 256), [0, 9, 70, 133, 254], [17]):
        s = torch.cuda.Stream()
        sg.set_cu_mask(ctx, s, cus)
        s.wait_stream(torch.cuda.current_stream())
        out, other = c.run(ctx, stream=s)
        assert torch.equal(out, want) and torch.equal(other, lse), cus
        sg.stream_release(ctx, s)


def test_pages_past_4_gib(ctx):
    c = Case([300, 40], [2, 5], 8, 8, 128, 64, torch.bfloat16, tree=True, seed=2)
    far = (6 << 30 >> c.shift)
    pool = torch.zeros(far * c.per, dtype=torch.bfloat16, device=DEV)
    table = c.table.copy()
    for r in range(2):
        for b in range(-(-c.totals[r] // c.block)):
            p, to = int(c.table[r, b]), far - 1 - 3 * int(c.table[r, b])
            pool[to * c.per:(to + 1) * c.per] = c.pool[p * c.per:(p + 1) * c.per].to(DEV)
            table[r, b] = to
    c.pages = far
    c.check(*c.run(ctx, table=table, pool=pool))
    assert ctx.device_error() == 0


def test_bad_pages_are_skipped_and_flagged(ctx):
    c = Case([100, 60], [2, 3], 4, 2, 64, 16, torch.float16, tree=False, seed=12)
    table = c.table.copy()
    table[0, 2] = c.pages
    out, lse = c.run(ctx, table=table)
    assert ctx.device_error() == sg.DEVERR_PT_RANGE
    # as if tokens 32..47 of request 0 were not there
    keep = [i for i in range(102) if i not in range(32, 48)]
    c.k[0], c.v[0], c.lens = c.k[0][keep], c.v[0][keep], [84, 60]
    c.check(out, lse)


def test_sequences_out_of_range_are_flagged(ctx):
    """Row starts past q, requests longer than max_nodes, lengths past the table:
    brought into range, nothing outside is written, and the flag is raised."""
    c = Case([20, 30], [3, 2], 4, 2, 64, 16, torch.bfloat16, tree=False, seed=13)
    c.run(ctx)
    pool, q, work, wide = c.keep
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    cache = sg.kv_cache(pool, c.pages, c.shift, 16, 2, 64, sg.BF16)
    sound = dict(q_start=[0, 3, 5], lens=[20, 30], totals=[23, 32])
    for bad in (dict(q_start=[0, 3, 9]), dict(q_start=[4, 3, 5]), dict(q_start=[0, 2 ** 31 - 1, 5]),
                dict(q_start=[0, 5, 5]), dict(lens=[24, 30]), dict(lens=[-1, 30]), dict(totals=[23, -7]),
                dict(totals=[23, 2 ** 31 - 1])):
        a = {k: i32(v) for k, v in {**sound, **bad}.items()}
        wide.fill_(7.0)
        sg.colored_tree_attention(ctx, cache, 0, q, a["q_start"], i32(c.table.tolist()), a["lens"], a["totals"],
                                  wide[:, 2:6], work, max_nodes=3)
        torch.cuda.synchronize()
        flags = ctx.device_error()
        assert flags & sg.DEVERR_SEQ, bad
        assert bool((wide[:, :2] == 7).all()) and bool((wide[:, 6:] == 7).all())


def test_graph_replays(ctx):
    """Captured once, replayed on new queries, keys and lengths, with other work between."""
    c = Case([700, 64], [4, 2], 4, 2, 128, 64, torch.bfloat16, tree=True, seed=21)
    c.run(ctx)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.call()
    for seed in (1, 2, 3):
        c.proj = torch.randn(c.proj.shape, generator=torch.Generator().manual_seed(seed)).to(c.dtype)
        c.q = c.proj[:, 1:1 + c.heads]
        c.keep[1].copy_(c.q)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        c.check(c.out.cpu(), c.d_lse.cpu())
        (torch.ones(1 << 20, device=DEV) * 2).sum().item()


def test_bindings_refuse_shapes_that_do_not_fit(ctx):
    c = Case([20, 30], [3, 2], 4, 2, 64, 16, torch.bfloat16, tree=True, seed=13)
    c.run(ctx)
    pool, q, work, wide = c.keep
    cache = sg.kv_cache(pool, c.pages, c.shift, 16, 2, 64, sg.BF16)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    a = dict(q=q, q_start=i32([0, 3, 5]), table=i32(c.table.tolist()), lens=i32([20, 30]), totals=i32([23, 32]),
             out=wide[:, 2:6], work=work, mask=c.mask.to(DEV))
    for name, bad in (("q", q[:4]), ("q", q.half()), ("out", wide), ("lens", i32([1])), ("q_start", i32([0, 5])),
                      ("mask", c.mask.to(DEV)[:4]), ("table", a["table"].long()),
                      ("lse", torch.zeros(5, 4, dtype=torch.float64, device=DEV))):
        with pytest.raises(ValueError):
            sg.colored_tree_attention(ctx, cache, 0, max_nodes=3, **{**a, name: bad})
    for kw in (dict(max_nodes=0), dict(scale=-1.0), dict(work=work[:256])):
        with pytest.raises(sg.SgdrcError):
            sg.colored_tree_attention(ctx, cache, 0, **{"max_nodes": 3, **a, **kw})
    torch.cuda.synchronize()
    ctx.device_error()
