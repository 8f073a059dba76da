"""Operators of a decoding step around the paged key/value cache, as cases
that can be timed.

Four kinds of call, in the order in which a program makes them: laying out
4-bit weights (``pack``, once), the product with such weights (``gemv``), the
write of new tokens to the cache with the norms and the position rotation of
queries and keys on the way (``rotate``), and the verification of drafted
tokens against the target's probabilities (``verify``).

4-bit weights: 16 rows by 128 columns are 1 KiB, [4 groups of lanes][16 rows]
of 16 bytes; word i of lane group g's piece holds columns 32 i + 8 g .. + 7,
column e at bits 4 (e / 2 + 4 (e % 2)).  All such blocks, [row tile][column
segment], then the scales, [row tile][segment][4][groups][4 rows], then the
zero points likewise; the whole lies in a pool's pages through a page table.

Where ``own`` is false the operators run in their plain form, elementary
torch operations; where it is true they are the package's calls.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_CTX = None


def _gemv(name, rows, cols, batch, group=128, dtype="bf16", zeros=False, shift=16):
    return {"name": name, "kind": "gemv", "rows": rows, "cols": cols, "batch": batch, "group": group, "dtype": dtype,
            "zeros": zeros, "shift": shift}


def _rotate(name, tokens, run, heads, kv, dim=128, block=64, dtype="bf16", rot=128, pairs=False, norm=True, far=4096):
    return {"name": name, "kind": "rotate", "tokens": tokens, "run": run, "heads": heads, "kv": kv, "dim": dim,
            "block": block, "dtype": dtype, "rot": rot, "pairs": pairs, "norm": norm, "far": far}


def _verify(name, requests, nodes, vocab, dtype="f32", draft=True, tree=False):
    return {"name": name, "kind": "verify", "requests": requests, "nodes_lo": nodes[0], "nodes_hi": nodes[1],
            "vocab": vocab, "dtype": dtype, "draft": draft, "tree": tree}


def listed():
    return [
        # odd sizes, where the call itself counts; the last columns do not fill a segment
        _gemv("gemv-small-b3-f16-zeros", 1003, 1056, 3, group=32, dtype="f16", zeros=True, shift=12),
        # the memory-bound layers of the benchmark: one token
        _gemv("gemv-down-b1", 4096, 11008, 1, shift=21),
        # a draft of eight nodes, zero points and small groups
        _gemv("gemv-up-b8-g32-zeros", 11008, 4096, 8, group=32, zeros=True),
        # a large layer, a draft of sixteen nodes
        _gemv("gemv-large-b16-g64", 32768, 8192, 16, group=64, shift=21),
        # the same layers laid out, as when a program starts
        {**_gemv("pack-small-f16-zeros", 1003, 1056, 1, group=32, dtype="f16", zeros=True, shift=12), "kind": "pack"},
        {**_gemv("pack-up", 11008, 4096, 1), "kind": "pack"},
        # one token each of 61 requests
        _rotate("rotate-61", 61, 1, 32, 8),
        # drafts of 24 nodes far into long documents, heads of 96 of which 64 dimensions turn, without norms
        _rotate("rotate-drafts-partial-f16", 1000, 24, 16, 4, dim=96, block=32, dtype="f16", rot=64, pairs=True,
                norm=False, far=900000),
        # prompts of about two thousand tokens each
        _rotate("rotate-prompts-16k", 16384, 2045, 32, 8),
        # one request's chain of five nodes: latency
        _verify("verify-1x5", 1, (5, 5), 32000),
        # trees of certain choices (the best tokens of a draft), half precision
        _verify("verify-32-trees-bf16", 32, (1, 48), 50257, dtype="bf16", draft=False, tree=True),
        # a full batch of sampled chains
        _verify("verify-64x8", 64, (8, 8), 131072),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["gemv", "gemv", "gemv", "gemv", "pack", "rotate", "rotate", "rotate", "verify", "verify",
                       "verify"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if kind in ("gemv", "pack"):
        group = rng.choice([32, 64, 128])
        rows = _log(rng, 16, 32768)
        most = min(16384, (1 << 28) // rows) if kind == "gemv" else min(16384, (11008 * 4096) // rows)
        cols = group * max(1, _log(rng, 64, max(most, 64)) // group)
        return {"kind": kind, "rows": rows, "cols": cols, "batch": rng.randint(1, 16) if kind == "gemv" else 1,
                "group": group, "dtype": dtype, "zeros": rng.random() < 0.4, "shift": rng.choice([12, 14, 16, 18, 21])}
    if kind == "rotate":
        kv, heads = rng.choice([(1, 8), (2, 14), (4, 16), (5, 15), (8, 8), (8, 32), (8, 64), (32, 32)])
        dim = rng.choice([64, 96, 128, 128, 128, 256])
        step = rng.random() < 0.4
        most = min(1024, (1 << 28) // (kv * dim * 128)) if step else (1 << 26) // ((heads + kv) * dim)
        return {"kind": kind, "tokens": _log(rng, 1, most), "run": 1 if step else _log(rng, 2, 4096), "heads": heads,
                "kv": kv, "dim": dim, "block": rng.choice([16, 32, 64, 64, 128]), "dtype": dtype,
                "rot": rng.choice([dim, dim, dim, dim // 2 // 16 * 16, 0]), "pairs": rng.random() < 0.4,
                "norm": rng.random() < 0.6, "far": _log(rng, 100, 1 << 20)}
    nodes = _log(rng, 1, 64)
    vocab = _log(rng, 1000, 262144)
    requests = _log(rng, 1, max(1, min(256, (1 << 26) // (nodes * vocab))))
    return {"kind": kind, "requests": requests, "nodes_lo": rng.choice([1, nodes]), "nodes_hi": nodes, "vocab": vocab,
            "dtype": rng.choice(["f32", "f32", "bf16", "f16"]), "draft": rng.random() < 0.6,
            "tree": nodes > 2 and rng.random() < 0.6}


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


def _parts(case):
    """Row tiles, column segments, groups of a segment, and bytes of the codes and of the scales."""
    tiles, segs, per = -(-case["rows"] // 16), -(-case["cols"] // 128), 128 // case["group"]
    return tiles, segs, per, tiles * segs * 1024, tiles * segs * per * 32


def _packed_bytes(case):
    _, _, _, codes, scales = _parts(case)
    return codes + scales * (2 if case["zeros"] else 1)


def _pages(case, g):
    """A pool of random bytes, and the page table of a tensor in it."""
    n = -(-_packed_bytes(case) >> case["shift"])
    pages = n + n // 4 + 3
    pool = torch.randint(-(1 << 31), 1 << 31, (pages << (case["shift"] - 2),), generator=g, device=DEV,
                         dtype=torch.int32)
    return pool.view(torch.uint8), _perm(pages, g)[:n].contiguous(), pages


def _scales(case, g):
    """Scales of trained-like weights (a few percent of outliers), and zero points."""
    n = case["cols"] // case["group"]
    s = (0.002 + 0.01 * torch.rand(case["rows"], n, generator=g, device=DEV)).to(DTYPES[case["dtype"]])
    z = torch.randint(4, 12, (case["rows"], n), generator=g, device=DEV).to(DTYPES[case["dtype"]])
    return s, z if case["zeros"] else None


def _scale_planes(case, s):
    """[rows, groups] in the layout of the tensor, with zeros where it is wider."""
    tiles, segs, per, _, _ = _parts(case)
    full = torch.zeros(tiles * 16, segs * per, dtype=s.dtype, device=DEV)
    full[:s.shape[0], :s.shape[1]] = s
    return full.view(tiles, 4, 4, segs, per).permute(0, 3, 1, 4, 2).contiguous().view(torch.uint8).flatten()


def _gemv_inputs(case, seed):
    """A tensor of random codes, already in its place."""
    g = _gen(seed)
    pool, table, pages = _pages(case, g)
    s, z = _scales(case, g)
    _, _, _, codes, scales = _parts(case)
    size = _packed_bytes(case)
    whole = pool.view(pages, -1)[table.long()].flatten()
    whole[codes:codes + scales] = _scale_planes(case, s)
    if z is not None:
        whole[codes + scales:size] = _scale_planes(case, z)
    pool.view(pages, -1)[table.long()] = whole.view(table.numel(), -1)
    x = torch.randn(case["batch"], case["cols"], generator=g, device=DEV).to(DTYPES[case["dtype"]])
    return {"pool": pool, "table": table, "pages": pages, "x": x}


def _pack_inputs(case, seed):
    g = _gen(seed)
    pool, table, pages = _pages(case, g)
    s, z = _scales(case, g)
    codes = torch.randint(0, 16, (case["rows"], case["cols"]), generator=g, device=DEV, dtype=torch.uint8)
    return {"pool": pool, "table": table, "pages": pages, "codes": codes, "scales": s, "zeros": z}


def _page(case):
    """Elements of a block of the cache, and the page size that holds it, as log2 of bytes."""
    elems = 2 * case["kv"] * case["block"] * case["dim"]
    return elems, max(10, (2 * elems - 1).bit_length())


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


def _rotate_inputs(case, seed):
    g, n, block = _gen(seed), case["tokens"], case["block"]
    runs = -(-n // case["run"])
    span = -(-(case["run"] + block) // block)  # blocks of a run that begins inside a block
    pages = runs * span + 1
    perm = _perm(pages, g).long()
    first = torch.randint(0, block, (runs,), generator=g, device=DEV)
    t = torch.arange(n, device=DEV)
    pos = first[t // case["run"]] + t % case["run"]
    slots = perm[t // case["run"] * span + pos // block] * block + pos % block
    # the place in the sequence: blocks before this run, as far as documents go
    before = torch.randint(0, case["far"], (runs,), generator=g, device=DEV)
    position = (before[t // case["run"]] + t % case["run"]).to(torch.int32)
    if runs > 1:  # the last request found no free pages, the first token of the one before is padding
        slots = torch.where(t // case["run"] == runs - 1, -1, slots)
        pad = t == (runs - 2) * case["run"]
        slots, position = torch.where(pad, -1, slots), torch.where(pad, -1, position).to(torch.int32)
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    dt = DTYPES[case["dtype"]]
    # queries, keys and values lie side by side in one projection's output
    proj = torch.randn(n, heads + 2 * kv, dim, generator=g, device=DEV).to(dt)
    half = case["rot"] // 2
    freq = (10000.0 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))).float().to(DEV)
    weights = [(1 + 0.1 * torch.randn(dim, generator=g, device=DEV)).to(dt) if case["norm"] else None
               for _ in range(2)]
    pool = torch.empty(pages << (_page(case)[1] - 1), dtype=dt, device=DEV).normal_(generator=g)
    return {"pool": pool, "pages": pages, "slots": slots, "position": position, "freq": freq if half else None,
            "q": proj[:, :heads], "k": proj[:, heads:heads + kv], "v": proj[:, heads + kv:], "q_norm": weights[0],
            "k_norm": weights[1]}


def _verify_inputs(case, seed):
    """Rows of the target's and the draft's probabilities, trees whose tokens
    were drawn from the draft's rows or are its best, and random numbers."""
    g, n, vocab = _gen(seed), case["requests"], case["vocab"]
    counts = _spread(case["nodes_lo"], case["nodes_hi"], n)
    order = torch.randperm(n, generator=g, device=DEV).tolist()
    counts = [counts[i] for i in order]
    starts = [0]
    for c in counts:
        starts.append(starts[-1] + c)
    tokens, most = starts[-1], case["nodes_hi"]
    q_start = _ints(starts)
    logits = 3.0 * torch.randn(tokens, vocab, generator=g, device=DEV)
    target = torch.softmax(logits, 1)
    logits += torch.randn(tokens, vocab, generator=g, device=DEV)
    guess = torch.softmax(logits, 1)
    del logits
    # parents: the node before, or one of the four before it
    node = torch.arange(most, device=DEV)
    back = torch.randint(0, 4, (n, most), generator=g, device=DEV) if case["tree"] else 0
    parent = (node - 1 - back).clamp(min=0).expand(n, most).clone()
    parent[:, 0] = -1
    has = node < _ints(counts)[:, None]
    row = (q_start[:-1, None] + parent.clamp(min=0)).clamp(max=tokens - 1).long()
    if case["draft"]:
        drawn = torch.multinomial(guess, 8, replacement=True, generator=g)
    else:
        drawn = guess.topk(8, 1).indices
    # a node takes the drawn or best token that its siblings before it left
    rank = ((parent[:, :, None] == parent[:, None, :]) & (node[None, :] < node[:, None])).sum(2).clamp(max=7)
    token = torch.gather(drawn[row.flatten()], 1, rank.view(-1, 1)).view(n, most)
    u = torch.rand(tokens, generator=g, device=DEV)
    lens = torch.randint(1, 1000, (n,), generator=g, device=DEV).to(torch.int32)
    totals = lens + _ints(counts)
    if n > 6:  # one of seven found no free pages
        totals = torch.where(torch.arange(n, device=DEV) % 7 == 6, lens, totals)
    dt = DTYPES[case["dtype"]]
    return {"target": target.to(dt), "draft": guess.to(dt) if case["draft"] else None,
            "tokens": token[has].to(torch.int32), "parents": parent[has].to(torch.int32), "u": u, "q_start": q_start,
            "lens": lens, "totals": totals}


INPUTS = {"gemv": _gemv_inputs, "pack": _pack_inputs, "rotate": _rotate_inputs, "verify": _verify_inputs}


def prepare(case, seed):
    st = INPUTS[case["kind"]](case, seed)
    st["case"] = case
    if case["kind"] == "gemv":
        st["y"] = torch.zeros(case["batch"], case["rows"], device=DEV)
    elif case["kind"] == "rotate":
        st["q_out"] = torch.zeros(st["q"].shape, dtype=st["q"].dtype, device=DEV)
    elif case["kind"] == "verify":
        n = case["requests"]
        st["path"] = torch.zeros(n, case["nodes_hi"], dtype=torch.int32, device=DEV)
        st["accepted"], st["next"] = (torch.zeros(n, dtype=torch.int32, device=DEV) for _ in range(2))
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
    if kind in ("gemv", "pack") and "w" not in st:  # a program keeps the descriptors of its weights
        dtype = {"bf16": sg.BF16, "f16": sg.F16}[case["dtype"]]
        st["w"] = sg.paged(st["pool"], st["table"], st["pages"])
        st["q4"] = sg.q4(case["rows"], case["cols"], case["group"], dtype, case["zeros"])
    if kind == "gemv":
        sg.colored_gemv_q4(ctx, st["w"], st["q4"], st["x"], case["batch"], st["y"], case["shift"])
        return st["y"]
    if kind == "pack":
        sg.colored_q4_pack(ctx, st["w"], st["q4"], st["codes"], st["scales"], st["zeros"], case["shift"])
        return st["pool"]
    if kind == "rotate":
        if "cache" not in st:
            st["cache"] = sg.kv_cache(st["pool"], st["pages"], _page(case)[1], case["block"], case["kv"], case["dim"],
                                      {"bf16": sg.BF16, "f16": sg.F16}[case["dtype"]])
        sg.colored_kv_append_rotated(ctx, st["cache"], 0, st["q"], st["k"], st["v"], st["q_out"], st["slots"],
                                     st["position"], freq=st["freq"], interleaved=case["pairs"],
                                     q_norm=st["q_norm"], k_norm=st["k_norm"], eps=1e-6)
        return {"q": st["q_out"], "pool": st["pool"]}
    sg.colored_draft_verify(ctx, st["target"], st["tokens"], st["parents"], st["u"], st["q_start"], st["path"],
                            st["accepted"], st["next"], draft=st["draft"], lens=st["lens"], totals=st["totals"],
                            max_nodes=case["nodes_hi"])
    return {"path": st["path"], "accepted": st["accepted"], "next": st["next"]}


# bit position / 4 of each of a word's eight columns
NIBBLE = [0, 4, 1, 5, 2, 6, 3, 7]


def _plain_gemv(st):
    case = st["case"]
    tiles, segs, per, codes, scales = _parts(case)
    whole = st["pool"].view(st["pages"], -1)[st["table"].long()].flatten()
    b = whole[:codes].view(tiles, segs, 4, 16, 4, 4)
    n = torch.stack([b & 15, b >> 4], -1).view(tiles, segs, 4, 16, 4, 8)[..., NIBBLE]
    n = n.permute(0, 3, 1, 4, 2, 5).reshape(tiles * 16, segs * per, case["group"]).float()

    def plane(at):
        p = whole[at:at + scales].view(DTYPES[case["dtype"]]).view(tiles, segs, 4, per, 4)
        return p.permute(0, 2, 4, 1, 3).reshape(tiles * 16, segs * per, 1).float()

    w = plane(codes) * (n - (plane(codes + scales) if case["zeros"] else 8.0))
    w = w.view(tiles * 16, -1)[:case["rows"], :case["cols"]]
    return torch.matmul(st["x"].float(), w.t())


def _plain_pack(st):
    case = st["case"]
    tiles, segs, per, codes, scales = _parts(case)
    n = torch.zeros(tiles * 16, segs * 128, dtype=torch.uint8, device=DEV)
    n[:case["rows"], :case["cols"]] = st["codes"]
    n = n.view(tiles, 16, segs, 4, 4, 8).permute(0, 2, 4, 1, 3, 5)  # [tile][segment][g][row][word][column]
    lo, hi = n[..., 0::2], n[..., 1::2]                             # nibbles 0..3 and 4..7
    b = torch.stack([lo[..., 0] | (lo[..., 1] << 4), lo[..., 2] | (lo[..., 3] << 4),
                     hi[..., 0] | (hi[..., 1] << 4), hi[..., 2] | (hi[..., 3] << 4)], -1)
    parts = [b.flatten()] + [_scale_planes(case, t) for t in (st["scales"], st["zeros"]) if t is not None]
    pool = st["pool"].view(st["pages"], -1)
    whole = pool[st["table"].long()].flatten()
    whole[:_packed_bytes(case)] = torch.cat(parts)
    pool[st["table"].long()] = whole.view(st["table"].numel(), -1)
    return st["pool"]


def _plain_rotate(st):
    case = st["case"]
    rot, half = case["rot"], case["rot"] // 2
    if rot:  # angles of far positions lose their fraction in 32 bits
        a = st["position"].double()[:, None] * st["freq"].double()
        cos, sin = torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]

    def turned(x, weight):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight.float()
        if rot:
            r = x[..., :rot]
            u, v = (r[..., 0::2], r[..., 1::2]) if case["pairs"] else (r[..., :half], r[..., half:])
            u, v = u * cos - v * sin, u * sin + v * cos
            r = torch.stack([u, v], -1).flatten(-2) if case["pairs"] else torch.cat([u, v], -1)
            x = torch.cat([r, x[..., rot:]], -1)
        return x.to(st["q"].dtype)

    there = st["position"] >= 0
    q = torch.where(there[:, None, None], turned(st["q"], st["q_norm"]), 0)
    ok = there & (st["slots"] >= 0)
    slots, block = st["slots"][ok], case["block"]
    page, off = slots // block, slots % block
    _k_part(case, st["pool"])[page, :, :, off] = turned(st["k"], st["k_norm"])[ok].unflatten(2, (-1, 8))
    _v_part(case, st["pool"])[page, :, off // 8, :, off % 8] = st["v"][ok]
    return {"q": q, "pool": st["pool"]}


def _plain_verify(st):
    """Node after node of all requests side by side: a request stands at a node,
    with the weights that are left there and their sum."""
    case, p, q = st["case"], st["target"], st["draft"]
    n, vocab, most = case["requests"], case["vocab"], case["nodes_hi"]
    start = st["q_start"][:-1].long()
    count = torch.where(st["totals"] - st["lens"] >= st["q_start"].diff(), st["q_start"].diff(), 0)
    cur, at = start.clamp(max=p.shape[0] - 1), torch.zeros_like(start)
    w, c = p[cur].double(), torch.zeros(n, dtype=torch.float64, device=DEV)
    path = torch.full((n, most), -1, dtype=torch.int32, device=DEV)
    path[:, 0] = torch.where(count > 0, 0, -1)
    depth = (count > 0).long()
    rows = torch.arange(n, device=DEV)
    s = torch.ones(n, dtype=torch.float64, device=DEV)
    for i in range(1, most):
        node = (start + i).clamp(max=p.shape[0] - 1)
        here = (i < count) & (st["parents"][node] == at)
        t = st["tokens"][node].long()
        left = w[rows, t]
        chance = q[cur, t].double() if q is not None else 1.0
        yes = here & (st["u"][node].double() * chance * s < left)
        no = here & ~yes
        if q is None:
            w[rows, t] = torch.where(no, 0.0, left)
        else:
            c = torch.where(no, c + s, c)
            w = torch.where(no[:, None], (p[cur].double() - c[:, None] * q[cur].double()).clamp(min=0), w)
        s = torch.where(no, w.sum(1), s)
        path[rows, depth.clamp(max=most - 1)] = torch.where(yes, i, path[rows, depth.clamp(max=most - 1)])
        depth = depth + yes
        at, cur = torch.where(yes, i, at), torch.where(yes, node, cur)
        w = torch.where(yes[:, None], p[cur].double(), w)
        c, s = torch.where(yes, 0.0, c), torch.where(yes, 1.0, s)
    w = torch.where(w.sum(1, keepdim=True) > 0, w, p[cur].double())
    run_sum = torch.cumsum(w, 1)
    goal = st["u"][start.clamp(max=p.shape[0] - 1)].double() * w.sum(1)
    past = run_sum > goal[:, None]
    last = vocab - 1 - (w > 0).flip(1).to(torch.int8).argmax(1)
    nxt = torch.where(past.any(1), past.to(torch.int8).argmax(1), last)
    return {"path": path, "accepted": depth.to(torch.int32), "next": torch.where(count > 0, nxt, -1).to(torch.int32)}


PLAIN = {"gemv": _plain_gemv, "pack": _plain_pack, "rotate": _plain_rotate, "verify": _plain_verify}


def work(case):
    kind = case["kind"]
    if kind in ("gemv", "pack"):
        m, k, b = case["rows"], case["cols"], case["batch"]
        scales = 2 * m * (k // case["group"]) * (2 if case["zeros"] else 1)
        if kind == "pack":
            return {"bytes": m * k + m * k // 2 + 2 * scales, "flops": 0}
        return {"bytes": m * k // 2 + scales + 2 * b * k + 4 * b * m, "flops": 2 * m * k * b}
    if kind == "rotate":
        heads, dim, n = case["heads"] + case["kv"], case["dim"], case["tokens"]
        # a norm is a square, a sum and two products, a rotation three operations an element
        return {"bytes": n * (4 * (heads + case["kv"]) * dim + 12),
                "flops": n * heads * (4 * dim * case["norm"] + 3 * case["rot"])}
    # a request reads the row that its next token comes from, and the draft's beside it
    n, es = case["requests"], 4 if case["dtype"] == "f32" else 2
    nodes = sum(_spread(case["nodes_lo"], case["nodes_hi"], n))
    rows = 2 if case["draft"] and case["nodes_hi"] > 1 else 1
    return {"bytes": n * (rows * case["vocab"] * es + 4 * case["nodes_hi"] + 20) + nodes * (12 + rows * es),
            "flops": n * case["vocab"] * rows}


# ------------------------------------------------------------- 64-bit values

def exact(case, seed):
    st = INPUTS[case["kind"]](case, seed)
    return {"gemv": _exact_gemv, "pack": _exact_pack, "rotate": _exact_rotate, "verify": _exact_verify}[
        case["kind"]](case, st)


def _at(case, st, where):
    """Byte addresses in the pool of the tensor's bytes ``where``."""
    shift = case["shift"]
    return (st["table"].long()[where >> shift] << shift) + (where & ((1 << shift) - 1))


def _code_bytes(case, rows, cols):
    """The tensor's byte that holds a code, and whether it is the upper half."""
    segs = _parts(case)[1]
    k, e = cols % 128, cols % 8
    nib = e // 2 + 4 * (e % 2)
    byte = ((rows // 16 * segs + cols // 128) * 1024 + (k % 32 // 8 * 16 + rows % 16) * 16 + k // 32 * 4 + nib // 2)
    return byte, nib % 2


def _scale_bytes(case, rows, groups):
    _, segs, per, codes, _ = _parts(case)
    r = rows % 16
    return codes + 2 * ((((rows // 16 * segs + groups // per) * 4 + r // 4) * per + groups % per) * 4 + r % 4)


def _exact_gemv(case, st):
    """Through the address of every weight, some rows at a time."""
    k, dt = torch.arange(case["cols"], device=DEV), DTYPES[case["dtype"]]
    x, out = st["x"].double(), []
    step = max(16, (1 << 24) // case["cols"])
    for m0 in range(0, case["rows"], step):
        m = torch.arange(m0, min(m0 + step, case["rows"]), device=DEV)[:, None]
        byte, upper = _code_bytes(case, m, k)
        n = (st["pool"][_at(case, st, byte)].long() >> (4 * upper)) & 15
        sb = _scale_bytes(case, m, torch.arange(case["cols"] // case["group"], device=DEV))
        half = st["pool"].view(dt)
        s = half[_at(case, st, sb) >> 1].double()
        z = half[_at(case, st, sb + _parts(case)[4]) >> 1].double() if case["zeros"] else torch.full_like(s, 8)
        w = s.repeat_interleave(case["group"], 1) * (n - z.repeat_interleave(case["group"], 1))
        out.append(x @ w.t().contiguous())
    return torch.cat(out, 1)


def _exact_pack(case, st):
    """Through the address of every code and scale."""
    tiles, segs, per, _, _ = _parts(case)
    pool = st["pool"].clone()
    m, k = torch.arange(tiles * 16, device=DEV)[:, None], torch.arange(segs * 128, device=DEV)
    codes = torch.nn.functional.pad(st["codes"], (0, segs * 128 - case["cols"], 0, tiles * 16 - case["rows"]))
    byte, upper = _code_bytes(case, m, k)
    byte = _at(case, st, byte)
    pool[byte[:, upper == 0]] = codes[:, upper == 0]
    pool[byte[:, upper == 1]] += codes[:, upper == 1] * 16
    half = pool.view(DTYPES[case["dtype"]])
    groups = torch.arange(segs * per, device=DEV)
    for i, t in enumerate((st["scales"], st["zeros"])):
        if t is not None:
            t = torch.nn.functional.pad(t, (0, segs * per - t.shape[1], 0, tiles * 16 - t.shape[0]))
            half[_at(case, st, _scale_bytes(case, m, groups) + i * _parts(case)[4]) >> 1] = t
    return pool


def _exact_rotate(case, st):
    """Rotations as products of complex numbers, through element addresses."""
    block, dim, rot = case["block"], case["dim"], case["rot"]
    per = 1 << (_page(case)[1] - 1)

    def turned(x, weight):
        x = x.double()
        if weight is not None:
            x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / dim + 1e-6) * weight.double()
        if rot:
            i = torch.arange(rot // 2, device=DEV)
            first, second = (2 * i, 2 * i + 1) if case["pairs"] else (i, i + rot // 2)
            angle = st["position"].double()[:, None, None] * st["freq"].double()
            z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.ones_like(angle), angle)
            x = x.clone()
            x[..., first], x[..., second] = z.real, z.imag
        return x

    q = turned(st["q"], st["q_norm"])
    q[st["position"] < 0] = 0
    pool = st["pool"].double()
    ok = (st["slots"] >= 0) & (st["position"] >= 0)
    slot = st["slots"][ok][:, None, None]
    h, d = torch.arange(case["kv"], device=DEV)[:, None], torch.arange(dim, device=DEV)
    base, tok = slot // block * per + h * 2 * block * dim, slot % block
    pool[base + (d // 8 * block + tok) * 8 + d % 8] = turned(st["k"], st["k_norm"])[ok]
    pool[base + block * dim + (tok // 8 * dim + d) * 8 + tok % 8] = st["v"][ok].double()
    return {"q": q, "pool": pool}


def _exact_verify(case, st):
    """Request after request, on the host, by the rule itself: a normalised
    distribution that a rejection replaces."""
    starts, u = st["q_start"].tolist(), st["u"].double().tolist()
    tokens, parents = st["tokens"].tolist(), st["parents"].tolist()
    grown = (st["totals"] - st["lens"]).tolist()
    paths, accepted, nxt = [], [], []

    def row(t, i):
        return t[i].double().cpu().numpy()

    for r in range(case["requests"]):
        a, n = starts[r], starts[r + 1] - starts[r]
        path = [0] if n and grown[r] >= n else []
        if path:
            left, total = row(st["target"], a), 1.0    # left / total is the distribution now
            scale = 0.0
            for i in range(1, n):
                if parents[a + i] != path[-1]:
                    continue
                t = tokens[a + i]
                guess = float(st["draft"][a + path[-1], t]) if case["draft"] else 1.0
                if u[a + i] * guess < left[t] / total if total > 0 else False:
                    path.append(i)
                    left, total, scale = row(st["target"], a + i), 1.0, 0.0
                elif case["draft"]:
                    scale += total
                    left = np.maximum(row(st["target"], a + path[-1]) - scale * row(st["draft"], a + path[-1]), 0)
                    total = float(left.sum())
                else:
                    left[t] = 0
                    total = float(left.sum())
            if left.sum() == 0:
                left = row(st["target"], a + path[-1])
            run_sum = np.cumsum(left)
            v = int(np.searchsorted(run_sum, u[a] * run_sum[-1], side="right"))
            nxt.append(v if v < len(left) else int(np.nonzero(left)[0][-1]))
        else:
            nxt.append(-1)
        accepted.append(len(path))
        paths.append(path + [-1] * (case["nodes_hi"] - len(path)))
    return {"path": _ints(paths), "accepted": _ints(accepted), "next": _ints(nxt)}
