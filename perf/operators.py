"""The operators of a paged key/value cache, as cases that can be timed.

Four kinds of call, in the order in which a decoding step makes them: the
block tables and slot maps of the step (``map``), the write of the new tokens
(``append``), the attention of drafted tokens over the cache (``attend``) and
the closing up of an accepted draft (``commit``).

The cache's layout is the one that the calls define: a pool page holds one
block of tokens of one layer, one chunk per key/value head, K as
[dim / 8][block][8 dims] and then V as [block / 8][dim][8 tokens].

Where ``own`` is false the operators run in their plain form, elementary
torch operations in 32 bits; where it is true they are the package's calls.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
_CTX = None


def _attend(name, requests, ctx, nodes, heads, kv, dim=128, block=64, dtype="bf16", cap=0.0, tree=False):
    return {"name": name, "kind": "attend", "requests": requests, "ctx_lo": ctx[0], "ctx_hi": ctx[1],
            "nodes_lo": nodes[0], "nodes_hi": nodes[1], "heads": heads, "kv": kv, "dim": dim, "block": block,
            "dtype": dtype, "cap": cap, "tree": tree}


def listed():
    return [
        # one decoding step of a few requests: every one gets one token
        {"name": "map-8", "kind": "map", "requests": 8, "block": 16, "len": 1500, "new": 1, "ended": 0,
         "short": False},
        # a busy server's step: drafts and prompt pieces, every ninth request
        # has ended, and the free pages do not reach for all
        {"name": "map-2048-short", "kind": "map", "requests": 2048, "block": 64, "len": 4000, "new": 32,
         "ended": 9, "short": True},
        # the new tokens of one decoding step
        {"name": "append-61", "kind": "append", "tokens": 61, "run": 1, "kv": 8, "dim": 128, "block": 64,
         "dtype": "bf16"},
        # prompts of about two thousand tokens each
        {"name": "append-prompts-16k", "kind": "append", "tokens": 16384, "run": 2045, "kv": 8, "dim": 128,
         "block": 64, "dtype": "bf16"},
        # four accepted tokens each of a few requests, in every layer of a small model
        {"name": "commit-7", "kind": "commit", "requests": 7, "layers": 12, "ctx": 300, "nodes": 24,
         "accepted": 4, "kv": 4, "dim": 64, "block": 32, "dtype": "f16"},
        # the same for a full batch of a larger one
        {"name": "commit-64", "kind": "commit", "requests": 64, "layers": 32, "ctx": 200, "nodes": 60,
         "accepted": 6, "kv": 8, "dim": 128, "block": 64, "dtype": "bf16"},
        # one sequence, one token: latency
        _attend("attend-1x1k", 1, (1009, 1009), (1, 1), 32, 8),
        # sixteen sequences with a head of keys for every query head (hidden size 4096)
        _attend("attend-16x4k-f16", 16, (301, 4096), (1, 1), 32, 32, block=16, dtype="f16"),
        # a full batch of single tokens over a cache of more than 4 GiB
        _attend("attend-96x24k", 96, (0, 24000), (1, 1), 32, 8),
        # one long document, a draft of two dozen nodes
        _attend("attend-tree24x128k", 1, (131001, 131001), (24, 24), 32, 8, tree=True),
        # ragged drafts with capped scores and wide heads; one request has nothing cached yet
        _attend("attend-tree-12x6k-cap", 12, (0, 6000), (1, 47), 16, 8, dim=256, block=32, cap=50.0, tree=True),
        # large drafts of a batch, eight query heads to a key head: arithmetic counts
        _attend("attend-tree64x24x8k", 24, (2000, 8000), (64, 64), 64, 8, tree=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["map", "append", "commit", "attend", "attend", "attend", "attend"])
    if kind == "map":
        return {"kind": kind, "requests": _log(rng, 1, 4096), "block": rng.choice([16, 32, 64, 128]),
                "len": _log(rng, 1, 8000), "new": _log(rng, 1, 64), "ended": rng.choice([0, 0, 5, 16]),
                "short": rng.random() < 0.25}
    kv, group = rng.choice([(1, 8), (2, 7), (4, 4), (5, 3), (8, 1), (8, 2), (8, 4), (8, 8), (32, 1)])
    dim, block = rng.choice([64, 96, 128, 128, 128, 256]), rng.choice([16, 32, 64, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if kind == "append":
        # single tokens, each in a block of its own request, or prompts
        step = rng.random() < 0.4
        tokens = _log(rng, 1, min(1024, (1 << 28) // (kv * dim * block)) if step else (1 << 24) // (kv * dim))
        return {"kind": kind, "tokens": tokens, "run": 1 if step else _log(rng, 2, 4096), "kv": kv, "dim": dim,
                "block": block, "dtype": dtype}
    if kind == "commit":
        nodes = _log(rng, 4, 64)
        return {"kind": kind, "requests": _log(rng, 1, 64 * 1024 // max(1024, kv * dim)),
                "layers": rng.randint(1, 32), "ctx": rng.randint(1, 300), "nodes": nodes,
                "accepted": rng.randint(1, min(8, nodes // 2)), "kv": kv, "dim": dim, "block": block,
                "dtype": dtype}
    requests = _log(rng, 1, 96)
    hi = _log(rng, 16, min(131072, 1100000 * 1024 // (requests * max(kv * dim, 1024))))
    nodes = 1 if rng.random() < 0.4 else _log(rng, 2, 64)
    # no more arithmetic than the largest listed case
    while requests * nodes * kv * group * hi * dim > 24 * 64 * 64 * 5000 * 128:
        nodes, hi = max(1, nodes // 2), hi if nodes > 1 else hi // 2
    return {"kind": kind, "requests": requests, "ctx_lo": rng.choice([0, hi // 16, hi // 2, hi]), "ctx_hi": hi,
            "nodes_lo": rng.choice([1, nodes]), "nodes_hi": nodes, "heads": kv * group, "kv": kv, "dim": dim,
            "block": block, "dtype": dtype, "cap": rng.choice([0.0, 0.0, 30.0]),
            "tree": nodes > 1 and rng.random() < 0.75}


# ---------------------------------------------------------------- inputs

def _ctx():
    """The package's context, one for the process."""
    global _CTX
    if _CTX is None:
        import paper_2407_13996_amd as sg
        _CTX = sg.Context(0)
    return _CTX


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly."""
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _perm(n, g):
    return torch.randperm(n, generator=g, device=DEV).to(torch.int32)


def _page(case):
    """Elements of a block of one layer, and the page size that holds it, as log2 of bytes."""
    elems = 2 * case["kv"] * case["block"] * case["dim"]
    return elems, max(10, (2 * elems - 1).bit_length())


def _cache(case, pages, g):
    """A pool of ``pages`` pages a layer with values in all of them."""
    shift = _page(case)[1]
    pool = torch.empty(case.get("layers", 1) * pages << (shift - 1), dtype=DTYPES[case["dtype"]], device=DEV)
    return pool.normal_(generator=g)


def _k_part(case, pool):
    """K of every page, [page][head][dim / 8][block][8]."""
    elems, shift = _page(case)
    half = case["block"] * case["dim"]
    chunks = pool.view(-1, 1 << (shift - 1))[:, :elems].view(-1, case["kv"], 2, half)
    return chunks[:, :, 0].unflatten(2, (case["dim"] // 8, case["block"], 8))


def _v_part(case, pool):
    """V of every page, [page][head][block / 8][dim][8]."""
    elems, shift = _page(case)
    half = case["block"] * case["dim"]
    chunks = pool.view(-1, 1 << (shift - 1))[:, :elems].view(-1, case["kv"], 2, half)
    return chunks[:, :, 1].unflatten(2, (case["block"] // 8, case["dim"], 8))


def _map_inputs(case, seed):
    """A server's state between two steps.  Some requests hold a block more
    than their tokens need, from a draft that was cut."""
    g, n, block = _gen(seed), case["requests"], case["block"]
    order = torch.randperm(n, generator=g, device=DEV)
    lens = _ints(_spread(0 if n > 1 else case["len"], case["len"], n))[order]
    new = _ints(_spread(min(1, case["new"]), case["new"], n))[torch.randperm(n, generator=g, device=DEV)]
    width = -(-(case["len"] + case["new"]) // block) + 1
    held = (lens + block - 1) // block
    held = held + torch.randint(0, 2, (n,), generator=g, device=DEV, dtype=torch.int32) * (held > 0)
    tokens = int(new.sum())  # the step's arrays are as long as if no request had ended
    if case["ended"]:
        new = torch.where(torch.arange(n, device=DEV) % case["ended"] == 0, -1, new).to(torch.int32)
    pages = n * width
    perm = _perm(pages, g)
    col = torch.arange(width, device=DEV)
    table = torch.full((n, width), -1, dtype=torch.int32, device=DEV)
    start = torch.cumsum(held, 0) - held
    mine = col < held[:, None]
    table = torch.where(mine, perm[(start[:, None] + col).clamp(max=pages - 1)], table).to(torch.int32)
    # the free pages wait in a ring; the counters have run for a while
    used = int(held.sum())
    free = pages - used
    if case["short"]:
        need = ((lens + new.clamp(min=0) + block - 1) // block - held).clamp(min=0)
        free = min(free, int(need.sum()) * 2 // 3)
    head = 7 * pages + int(torch.randint(0, pages, (1,), generator=g, device=DEV))
    ring = torch.full((pages,), -1, dtype=torch.int32, device=DEV)
    ring[(head + torch.arange(free, device=DEV)) % pages] = perm[used:used + free]
    return {"lens": lens, "new": new, "held": held, "table": table, "ring": ring,
            "state": torch.tensor([head, head + free], dtype=torch.int64, device=DEV), "tokens": tokens}


def _append_inputs(case, seed):
    g, n, block = _gen(seed), case["tokens"], case["block"]
    runs = -(-n // case["run"])
    span = -(-(case["run"] + block) // block)  # blocks of a run that begins inside a block
    pages = runs * span + 1
    perm = _perm(pages, g).long()
    first = torch.randint(0, block, (runs,), generator=g, device=DEV)
    t = torch.arange(n, device=DEV)
    pos = first[t // case["run"]] + t % case["run"]
    slots = perm[t // case["run"] * span + pos // block] * block + pos % block
    if runs > 1:  # the last request found no free pages
        slots = torch.where(t // case["run"] == runs - 1, -1, slots)
    kv, dim = case["kv"], case["dim"]
    # keys and values lie beside the queries in one projection's output
    proj = torch.randn(n, 3 * kv, dim, generator=g, device=DEV).to(DTYPES[case["dtype"]])
    return {"pool": _cache(case, pages, g), "pages": pages, "slots": slots, "k": proj[:, kv:2 * kv],
            "v": proj[:, 2 * kv:]}


def _commit_inputs(case, seed):
    g, n, block, nodes, acc = _gen(seed), case["requests"], case["block"], case["nodes"], case["accepted"]
    width = -(-(case["ctx"] + nodes) // block)
    pages = n * width + 3
    table = _perm(pages, g)[:n * width].view(n, width)
    lens = _ints(_spread(case["ctx"] // 2, case["ctx"], n))[torch.randperm(n, generator=g, device=DEV)]
    # a path through a broad tree: the root, then nodes past the accepted count
    rest = torch.rand(n, nodes - acc, generator=g, device=DEV).argsort(1)[:, :acc - 1].sort(1).values + acc
    path = torch.cat([torch.zeros(n, 1, dtype=torch.int64, device=DEV), rest], 1).to(torch.int32)
    return {"pool": _cache(case, pages, g), "pages": pages, "table": table.contiguous(), "lens": lens,
            "path": path.contiguous(), "accepted": torch.full((n,), acc, dtype=torch.int32, device=DEV)}


def _masks(counts, words, g):
    """Rows of visible nodes, a bit each, of random trees (a node's parent is
    one of the eight before it); a tree's last node of four or more is padding
    that sees nothing."""
    n, most = len(counts), max(counts)
    parent = (torch.arange(most, device=DEV) - 1
              - torch.randint(0, 8, (n, most), generator=g, device=DEV)).clamp(min=0)
    vis = torch.eye(most, dtype=torch.bool, device=DEV).expand(n, most, most).clone()
    for i in range(1, most):
        vis[:, i] |= vis[torch.arange(n, device=DEV), parent[:, i]]
    rows = torch.cat([vis[r, :c] & ((torch.arange(c, device=DEV) < c - 1) | (c < 4))[:, None]
                      for r, c in enumerate(counts)])
    rows = torch.nn.functional.pad(rows, (0, 64 * words - most)).view(-1, words, 64)
    return (rows.long() << torch.arange(64, device=DEV)).sum(2)


def _attend_inputs(case, seed):
    g, n, block = _gen(seed), case["requests"], case["block"]
    order = torch.randperm(n, generator=g, device=DEV).tolist()
    lens = _spread(case["ctx_lo"], case["ctx_hi"], n)
    counts = _spread(case["nodes_lo"], case["nodes_hi"], n)[::-1]
    lens, counts = [lens[i] for i in order], [counts[i] for i in order]
    totals = [a + b for a, b in zip(lens, counts)]
    used = [-(-t // block) for t in totals]
    width, pages = max(used) + 1, sum(used) + 5
    perm = _perm(pages, g)
    col, first = torch.arange(width, device=DEV), torch.cumsum(_ints(used), 0) - _ints(used)
    table = torch.where(col < _ints(used)[:, None], perm[(first[:, None] + col).clamp(max=pages - 1)], -1)
    starts = [0]
    for c in counts:
        starts.append(starts[-1] + c)
    tokens, heads, kv, dim = starts[-1], case["heads"], case["kv"], case["dim"]
    proj = torch.randn(tokens, heads + 2 * kv, dim, generator=g, device=DEV).to(DTYPES[case["dtype"]])
    words = -(-case["nodes_hi"] // 64)
    return {"pool": _cache(case, pages, g), "pages": pages, "table": table.to(torch.int32).contiguous(),
            "lens": _ints(lens), "totals": _ints(totals), "q_start": _ints(starts), "q": proj[:, :heads],
            "mask": _masks(counts, words, g) if case["tree"] else None, "longest": max(totals)}


INPUTS = {"map": _map_inputs, "append": _append_inputs, "commit": _commit_inputs, "attend": _attend_inputs}


def prepare(case, seed):
    st = INPUTS[case["kind"]](case, seed)
    st["case"] = case
    if case["kind"] == "map":
        n, tokens = case["requests"], st["tokens"]
        st["out"] = {"state": torch.zeros(2, dtype=torch.int64, device=DEV),
                     "held": torch.zeros(n, dtype=torch.int32, device=DEV),
                     "lens": torch.zeros(n, dtype=torch.int32, device=DEV),
                     "q_start": torch.zeros(n + 1, dtype=torch.int32, device=DEV),
                     "slots": torch.zeros(tokens, dtype=torch.int64, device=DEV),
                     "request": torch.zeros(tokens, dtype=torch.int32, device=DEV),
                     "position": torch.zeros(tokens, dtype=torch.int32, device=DEV)}
    elif case["kind"] == "commit":
        st["out"] = torch.zeros_like(st["lens"])
    elif case["kind"] == "attend":
        q = st["q"]
        st["o"] = torch.zeros(q.shape, dtype=q.dtype, device=DEV)
        st["lse"] = torch.zeros(q.shape[:2], device=DEV)
    return st


# ------------------------------------------------------------------ calls

def run(st):
    kind = st["case"]["kind"]
    if own:
        return _own(st, kind)
    return PLAIN[kind](st)


def _own(st, kind):
    import paper_2407_13996_amd as sg
    case, ctx = st["case"], _ctx()
    if kind == "map":
        o = st["out"]
        sg.colored_kv_map(ctx, case["block"], st["ring"], st["state"], st["held"], st["lens"], st["new"],
                          st["table"], o["state"], o["held"], o["lens"], o["q_start"], o["slots"], o["request"],
                          o["position"])
        return {"table": st["table"], "ring": st["ring"], **o}
    if "cache" not in st:  # a program keeps the descriptor of its cache, and the workspace
        layers, shift = case.get("layers", 1), _page(case)[1]
        st["cache"] = sg.kv_cache(st["pool"], st["pages"], shift, case["block"], case["kv"], case["dim"],
                                  {"bf16": sg.BF16, "f16": sg.F16}[case["dtype"]], layers, st["pages"] << shift)
        if kind == "attend":
            size = sg.tree_attention_workspace(st["cache"], case["heads"], case["nodes_hi"])
            st["work"] = torch.empty(size, dtype=torch.uint8, device=DEV)
    if kind == "append":
        sg.colored_kv_append(ctx, st["cache"], 0, st["k"], st["v"], st["slots"])
        return st["pool"]
    if kind == "commit":
        sg.colored_kv_commit(ctx, st["cache"], st["table"], st["lens"], st["path"], st["accepted"], st["out"])
        return {"pool": st["pool"], "lens": st["out"]}
    sg.colored_tree_attention(ctx, st["cache"], 0, st["q"], st["q_start"], st["table"], st["lens"], st["totals"],
                              st["o"], st["work"], lse=st["lse"], mask=st["mask"], max_nodes=case["nodes_hi"],
                              scale=case["dim"] ** -0.5, softcap=case["cap"])
    return {"o": st["o"], "lse": st["lse"]}


def _plain_map(st):
    block, table, ring, lens, held = st["case"]["block"], st["table"], st["ring"], st["lens"], st["held"]
    n, width = table.shape
    head, tail = st["state"][0], st["state"][1]
    ended = st["new"] < 0
    new = st["new"].clamp(min=0)
    need = torch.where(ended, 0, ((lens + new + block - 1) // block - held).clamp(min=0))
    end = torch.cumsum(need, 0)
    served = ~ended & ((need == 0) | (end <= tail - head))
    taken = torch.where(served & (need > 0), end, 0).amax()
    col = torch.arange(width, device=DEV)
    # the table's new entries
    fresh = served[:, None] & (col >= held[:, None]) & (col < (held + need)[:, None])
    at = (head + (end - need - held)[:, None] + col) % ring.numel()
    table.copy_(torch.where(fresh, ring[at], table))
    # ended requests give their pages back
    freed = torch.where(ended, held, 0)
    back = torch.cumsum(freed, 0) - freed
    gone = ended[:, None] & (col < held[:, None])
    to = (tail + back[:, None] + col) % ring.numel()
    ring[to[gone]] = table[gone]
    q_start = torch.nn.functional.pad(torch.cumsum(new, 0), (1, 0))
    t = torch.arange(st["tokens"], device=DEV)
    real = t < q_start[-1]
    r = torch.searchsorted(q_start[1:], t, right=True).clamp(max=n - 1)
    pos = torch.where(real, lens[r] + t - q_start[r], 0)
    slots = (table[r, pos // block].long() & 0xFFFFFFFF) * block + pos % block
    o = {"state": torch.stack([head + taken, tail + freed.sum()]),
         "held": torch.where(ended, 0, torch.where(served, held + need, held)).to(torch.int32),
         "lens": torch.where(ended, 0, torch.where(served, lens + new, lens)).to(torch.int32),
         "q_start": q_start.to(torch.int32), "slots": torch.where(served[r] & real, slots, -1),
         "request": torch.where(real, r, -1).to(torch.int32),
         "position": torch.where(real, pos, -1).to(torch.int32)}
    return {"table": table, "ring": ring, **o}


def _plain_append(st):
    case = st["case"]
    ok = st["slots"] >= 0
    slots, block = st["slots"][ok], case["block"]
    page, off = slots // block, slots % block
    _k_part(case, st["pool"])[page, :, :, off] = st["k"][ok].unflatten(2, (-1, 8))
    _v_part(case, st["pool"])[page, :, off // 8, :, off % 8] = st["v"][ok]
    return st["pool"]


def _plain_commit(st):
    case, block = st["case"], st["case"]["block"]
    layer = torch.arange(case["layers"], device=DEV)[:, None, None] * st["pages"]

    def at(node):
        pos = (st["lens"][:, None] + node).long()
        return layer + torch.gather(st["table"], 1, pos // block), (pos % block).expand(case["layers"], -1, -1)

    i = torch.arange(st["path"].shape[1], device=DEV)
    (sp, so), (dp, do) = at(st["path"]), at(i.expand(st["path"].shape))
    k, v = _k_part(case, st["pool"]), _v_part(case, st["pool"])
    k[dp, :, :, do] = k[sp, :, :, so]
    v[dp, :, do // 8, :, do % 8] = v[sp, :, so // 8, :, so % 8]
    return {"pool": st["pool"], "lens": st["lens"] + st["accepted"]}


def _plain_attend(st):
    case, table, q = st["case"], st["table"], st["q"]
    block, kv, dim, n = case["block"], case["kv"], case["dim"], case["requests"]
    group, most = case["heads"] // kv, case["nodes_hi"]
    pages = table[:, :-(-st["longest"] // block)].clamp(min=0).long()
    long = pages.shape[1] * block
    lens, totals, q_start = st["lens"].long(), st["totals"].long(), st["q_start"].long()
    pos = torch.arange(long, device=DEV)
    valid = (pos < totals[:, None])[:, None, :, None]
    k = _k_part(case, st["pool"])[pages].permute(0, 2, 1, 4, 3, 5).reshape(n, kv, long, dim)
    k = torch.where(valid, k, 0).float()
    v = _v_part(case, st["pool"])[pages].permute(0, 2, 1, 3, 5, 4).reshape(n, kv, long, dim)
    v = torch.where(valid, v, 0).float()
    tokens = q.shape[0]
    node = torch.arange(most, device=DEV)
    at = (q_start[:-1, None] + node).clamp(max=tokens - 1)
    qs = q.float()[at].view(n, most, kv, group, dim).transpose(1, 2).reshape(n, kv, most * group, dim)
    s = torch.matmul(qs, k.transpose(2, 3).contiguous()) * case["dim"] ** -0.5
    if case["cap"]:
        s = torch.tanh(s / case["cap"]) * case["cap"]
    j = (pos - lens[:, None])[:, None, :].expand(n, most, long)
    if st["mask"] is None:
        seen = j <= node[:, None]
    else:
        bits = ((st["mask"][:, :, None] >> torch.arange(64, device=DEV)) & 1).flatten(1).bool()
        seen = (j < 0) | torch.gather(bits[at], 2, j.clamp(0, bits.shape[1] - 1))
    seen = (seen & (pos < totals[:, None])[:, None]).repeat_interleave(group, 1)[:, None]
    s = torch.where(seen, s, -math.inf)
    m = s.amax(3, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, 0, m))
    l = p.sum(3, keepdim=True)
    o = torch.where(l > 0, torch.matmul(p, v) / l, 0)
    lse = torch.where(l > 0, m + torch.log(l), -math.inf)[..., 0]
    t = torch.arange(tokens, device=DEV)
    r = torch.searchsorted(q_start[1:], t, right=True)
    i = t - q_start[r]
    o = o.view(n, kv, most, group, dim).transpose(1, 2).reshape(n, most, kv * group, dim)
    lse = lse.view(n, kv, most, group).transpose(1, 2).reshape(n, most, kv * group)
    return {"o": o[r, i].to(q.dtype), "lse": lse[r, i]}


PLAIN = {"map": _plain_map, "append": _plain_append, "commit": _plain_commit, "attend": _plain_attend}


def work(case):
    if case["kind"] == "map":
        n = case["requests"]
        tokens = sum(_spread(min(1, case["new"]), case["new"], n))
        # lengths, new tokens and held blocks in and out, the starts, a page a
        # block, and slot, request and position of each token
        return {"bytes": 28 * n + 8 * (tokens // case["block"]) + 16 * tokens + 32, "flops": 0}
    token = 2 * case["kv"] * case["dim"] * 2  # a token's bytes in one layer
    if case["kind"] == "append":
        return {"bytes": case["tokens"] * (2 * token + 8), "flops": 0}
    if case["kind"] == "commit":
        moved = case["requests"] * (case["accepted"] - 1)
        return {"bytes": 2 * moved * case["layers"] * token + case["requests"] * (4 * case["accepted"] + 12) + 8,
                "flops": 0}
    n = case["requests"]
    lens = _spread(case["ctx_lo"], case["ctx_hi"], n)
    counts = _spread(case["nodes_lo"], case["nodes_hi"], n)[::-1]
    keys, rows = sum(lens) + sum(counts), sum(counts) * case["heads"]
    dots = sum(c * (a + (c + 1) / 2) for a, c in zip(lens, counts)) * case["heads"]
    return {"bytes": keys * token + rows * (4 * case["dim"] + 4) + 4 * keys // case["block"] + 12 * n
            + (8 * sum(counts) if case["tree"] else 0), "flops": 4 * case["dim"] * dots}


# ------------------------------------------------------------- 64-bit values

def exact(case, seed):
    st = INPUTS[case["kind"]](case, seed)
    return {"map": _exact_map, "append": _exact_append, "commit": _exact_commit, "attend": _exact_attend}[
        case["kind"]](case, st)


def _exact_map(case, st):
    """Request after request, on the host."""
    block, size = case["block"], st["ring"].numel()
    table, ring = [r.tolist() for r in st["table"]], st["ring"].tolist()
    head, tail = st["state"].tolist()
    begin, back, want, taken = head, tail, 0, 0
    held, lens, starts, slots, request, position = [], [], [0], [], [], []
    for r, (n, new, h) in enumerate(zip(st["lens"].tolist(), st["new"].tolist(), st["held"].tolist())):
        starts.append(starts[-1] + max(new, 0))
        if new < 0:
            for b in range(h):
                ring[back % size] = table[r][b]
                back += 1
            held.append(0)
            lens.append(0)
            continue
        need = max(0, -(-(n + new) // block) - h)
        ok = need == 0 or want + need <= tail - begin
        for b in range(need if ok else 0):
            table[r][h + b] = ring[(begin + want + b) % size]
        want += need
        taken = want if ok and need else taken
        held.append(h + need if ok else h)
        lens.append(n + new if ok else n)
        for p in range(n, n + new):
            slots.append(table[r][p // block] * block + p % block if ok else -1)
            request.append(r)
            position.append(p)
    for column in (slots, request, position):
        column += [-1] * (st["tokens"] - len(column))
    return {"table": _ints(table), "ring": _ints(ring), "state": torch.tensor([begin + taken, back], device=DEV),
            "held": _ints(held), "lens": _ints(lens), "q_start": _ints(starts),
            "slots": torch.tensor(slots, dtype=torch.int64, device=DEV), "request": _ints(request),
            "position": _ints(position)}


def _exact_append(case, st):
    """Through the byte address of every element."""
    block, dim, heads = case["block"], case["dim"], case["kv"]
    pool = st["pool"]
    per = 1 << (_page(case)[1] - 1)
    slot = st["slots"][:, None, None]
    h = torch.arange(heads, device=DEV)[:, None]
    d = torch.arange(dim, device=DEV)
    base = slot // block * per + h * 2 * block * dim
    tok = slot % block
    ka = base + (d // 8 * block + tok) * 8 + d % 8
    va = base + block * dim + (tok // 8 * dim + d) * 8 + tok % 8
    ok = (slot >= 0).expand_as(ka)
    pool[ka[ok]] = st["k"][ok]
    pool[va[ok]] = st["v"][ok]
    return pool


def _exact_commit(case, st):
    """Token after token of the path, through element addresses."""
    block, dim, heads = case["block"], case["dim"], case["kv"]
    per = 1 << (_page(case)[1] - 1)
    pool, table = st["pool"], st["table"].long()
    l = torch.arange(case["layers"], device=DEV)[:, None, None] * st["pages"]
    h = torch.arange(heads, device=DEV)[:, None]
    d = torch.arange(dim, device=DEV)
    rows = torch.arange(case["requests"], device=DEV)

    def where(pos):
        base = (l[None] + table[rows, pos // block][:, None, None, None]) * per + h * 2 * block * dim
        tok = (pos % block)[:, None, None, None]
        return (base + (d // 8 * block + tok) * 8 + d % 8,
                base + block * dim + (tok // 8 * dim + d) * 8 + tok % 8)

    for i in range(case["accepted"]):
        src, dst = where(st["lens"].long() + st["path"][:, i]), where(st["lens"].long() + i)
        for a, b in zip(src, dst):
            pool[b] = pool[a]
    return {"pool": pool, "lens": st["lens"] + st["accepted"]}


def _exact_attend(case, st):
    """A request at a time, in 64 bits."""
    kv, dim, block = case["kv"], case["dim"], case["block"]
    group = case["heads"] // kv
    o, lse = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV), []
    starts, lens, totals = (st[x].tolist() for x in ("q_start", "lens", "totals"))
    for r, (a, c, t) in enumerate(zip(starts, lens, totals)):
        n = starts[r + 1] - a
        page = st["table"][r, :-(-t // block)].long()
        k = _k_part(case, st["pool"])[page].double().permute(1, 0, 3, 2, 4).reshape(kv, -1, dim)[:, :t]
        v = _v_part(case, st["pool"])[page].double().permute(1, 0, 2, 4, 3).reshape(kv, -1, dim)[:, :t]
        q = st["q"][a:a + n].double().view(n, kv, group, dim)
        seen = torch.ones(n, t, dtype=torch.bool, device=DEV)
        for i in range(n):
            if st["mask"] is None:
                seen[i, c + i + 1:] = False
            else:
                row = torch.arange(t - c, device=DEV)
                seen[i, c:] = (st["mask"][a + i][row // 64] >> (row % 64)) & 1 != 0
        for h in range(kv):
            s = q[:, h].reshape(n * group, dim) @ k[h].t().contiguous() / math.sqrt(dim)
            s = case["cap"] * torch.tanh(s / case["cap"]) if case["cap"] else s
            s = s.masked_fill(~seen.repeat_interleave(group, 0), -math.inf)
            top = torch.logsumexp(s, 1, keepdim=True)
            w = torch.where(top == -math.inf, 0.0, torch.exp(s - top))
            o[a:a + n, h * group:(h + 1) * group] = (w @ v[h]).view(n, group, dim)
            lse.append(top.view(n, group))
    each, at = [], 0
    for _ in starts[1:]:
        each.append(torch.cat(lse[at:at + kv], 1))
        at += kv
    return {"o": o, "lse": torch.cat(each)}
