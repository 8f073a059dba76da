"""Decoding with drafted trees over a key/value cache on chosen colours.

A small decoder with random weights serves several prompts at once.  The
weights and the cache's pages lie on pages of chosen colours; the pages that the
page table names become the ring of free pages of the cache.  Every step

* drafts a tree of tokens for each request from what followed its last token
  before (a chain, and another first guess beside it),
* gives the requests pages and the tokens slots (colored_kv_map),
* runs the layers: projections (colored_gemv), writes to the cache
  (colored_kv_append), attention of the tree's nodes (colored_tree_attention),
* walks down each tree as far as the model's own choices go, and closes the
  accepted path up in the cache (colored_kv_commit).

A prompt is a chain whose nodes are all accepted.  A request for which the ring has
too few pages accepts nothing and tries again in the next step; one that has
its tokens ends, and its pages go to the others.  Run on an MI355X:

    python examples/draft_decoding.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2407_13996_amd as sg  # noqa: E402

DEV = "cuda:0"
LAYERS, HIDDEN, HEADS, KV, DIM, VOCAB = 2, 256, 8, 2, 64, 384
BLOCK, SHIFT = 16, 14                 # tokens of a block, log2 of a page's bytes (both layers' blocks)
MASKS = [(1 << 14) | (1 << 19), (1 << 15) | (1 << 18)]   # four colours of 16 KiB pages
COLOURS = (1, 2)
ORIGIN = 1 << 40
MOST = 256                            # nodes of a request at most


class Weights:
    """Random weights, the matrices stored on pages of the chosen colours."""

    def __init__(self, ctx, seed):
        g = torch.Generator().manual_seed(seed)

        def normal(*shape, scale=1.0):
            return (torch.randn(*shape, generator=g) * scale).to(torch.bfloat16).to(DEV)

        self.embed = normal(VOCAB, HIDDEN)
        self.place = normal(1024, HIDDEN, scale=0.02)
        self.plain, self.paged = {}, {}
        for name, rows in [("logits", VOCAB)] + [(f"{n}{l}", r) for l in range(LAYERS)
                                                 for n, r in (("qkv", (HEADS + 2 * KV) * DIM), ("out", HIDDEN))]:
            k = HEADS * DIM if name.startswith("out") else HIDDEN
            w = normal(rows, k, scale=k ** -0.5)
            self.plain[name], self.paged[name] = w, coloured_copy(ctx, w)

    def apply(self, ctx, name, x):
        """x @ W^T in fp32, eight tokens a call."""
        w, (rows, k) = self.paged[name], self.plain[name].shape
        x = x.to(torch.bfloat16).contiguous()
        y = torch.empty(x.shape[0], rows, dtype=torch.float32, device=DEV)
        for t in range(0, x.shape[0], 8):
            n = min(8, x.shape[0] - t)
            sg.colored_gemv(ctx, w, sg.BF16, rows, k, x[t:], sg.BF16, n, y[t:], SHIFT)
        return y


def coloured_pages(ctx, n):
    """A pool with ``n`` pages of the chosen colours, and their numbers."""
    pages = 4 * n + 64
    table = torch.empty(n, dtype=torch.int32, device=DEV)
    sg.colour_alloc_pagetable(ctx, MASKS, ORIGIN, SHIFT, pages, COLOURS, n, table)
    return torch.zeros(pages << SHIFT, dtype=torch.uint8, device=DEV), table, pages


def coloured_copy(ctx, w):
    n = -(-w.numel() * w.element_size() // (1 << SHIFT))
    pool, table, pages = coloured_pages(ctx, n)
    to = sg.paged(pool, table, pages)
    sg.bimodal_relayout(ctx, to, sg.paged(w, torch.arange(n, dtype=torch.int32, device=DEV), n),
                        w.numel() * w.element_size(), SHIFT)
    return to


def norm(x):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-5)


def masks_and_depths(trees):
    """The nodes that each node of the trees sees (its ancestors and itself), as
    words of bits, and how far below the root it is."""
    words, depth = [], []
    for _, parents in trees:
        rows = []
        for i, p in enumerate(parents):
            rows.append((rows[p] if p >= 0 else 0) | 1 << i)
            depth.append(bin(rows[-1]).count("1") - 1)
        words += [[(r >> 64 * k) & (1 << 64) - 1 for k in range(MOST // 64)] for r in rows]
    return torch.tensor([[x - (1 << 64) if x >> 63 else x for x in row] for row in words], dtype=torch.int64,
                        device=DEV), depth


class Server:
    """The requests' state: the cache, its block tables and the free pages."""

    def __init__(self, ctx, weights, requests, most_tokens, blocks=None):
        self.ctx, self.w, self.n = ctx, weights, requests
        width = -(-most_tokens // BLOCK)
        self.pool, free, pages = coloured_pages(ctx, requests * width if blocks is None else blocks)
        self.ring = free.clone()      # all pages are free: the ring is the page table
        self.cache = sg.kv_cache(self.pool, pages, SHIFT, BLOCK, KV, DIM, sg.BF16, LAYERS, (1 << SHIFT) // LAYERS)
        self.ring_pos = torch.tensor([0, self.ring.numel()], dtype=torch.int64, device=DEV)
        self.held = torch.zeros(requests, dtype=torch.int32, device=DEV)
        self.lens = torch.zeros_like(self.held)
        self.table = torch.zeros(requests, width, dtype=torch.int32, device=DEV)
        self.work = torch.empty(sg.tree_attention_workspace(self.cache, HEADS, MOST), dtype=torch.uint8, device=DEV)

    def map(self, new, tokens):
        """Pages and slots for new[r] tokens of each request (-1: it ends)."""
        new = torch.tensor(new, dtype=torch.int32, device=DEV)
        pos, held, totals = (torch.empty_like(t) for t in (self.ring_pos, self.held, self.lens))
        q_start = torch.empty(self.n + 1, dtype=torch.int32, device=DEV)
        slots = torch.empty(tokens, dtype=torch.int64, device=DEV)
        request, position = (torch.empty(tokens, dtype=torch.int32, device=DEV) for _ in range(2))
        sg.colored_kv_map(self.ctx, BLOCK, self.ring, self.ring_pos, self.held, self.lens, new, self.table, pos, held,
                          totals, q_start, slots, request, position)
        self.ring_pos, self.held = pos, held
        return totals, q_start, slots

    def step(self, trees):
        """The model's next token after every node of every request's tree;
        trees[r]: (tokens, parents), a parent before its children, -1 the root's;
        None: the request ends.  None for a request that found no pages."""
        new = [-1 if t is None else len(t[0]) for t in trees]
        trees = [t or ([], []) for t in trees]
        counts = [len(t) for t, _ in trees]
        n = sum(counts)
        tokens = torch.tensor([t for tree, _ in trees for t in tree], device=DEV)
        mask, depth = masks_and_depths(trees)
        self.totals, q_start, slots = self.map(new, n)
        at = self.lens.repeat_interleave(torch.tensor(counts, device=DEV)).long() + torch.tensor(depth, device=DEV)
        x = self.w.embed[tokens].float() + self.w.place[at].float()
        for layer in range(LAYERS):
            qkv = self.w.apply(self.ctx, f"qkv{layer}", norm(x)).to(torch.bfloat16).view(n, HEADS + 2 * KV, DIM)
            q, k, v = qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV], qkv[:, HEADS + KV:]
            sg.colored_kv_append(self.ctx, self.cache, layer, k, v, slots)
            o = torch.empty(n, HEADS, DIM, dtype=torch.bfloat16, device=DEV)
            sg.colored_tree_attention(self.ctx, self.cache, layer, q, q_start, self.table, self.lens, self.totals, o,
                                      self.work, mask=mask, max_nodes=MOST, scale=DIM ** -0.5)
            x = x + self.w.apply(self.ctx, f"out{layer}", o.view(n, HEADS * DIM))
        best = self.w.apply(self.ctx, "logits", norm(x)).argmax(1).tolist()
        grown = (self.totals - self.lens).tolist()
        return [best[sum(counts[:r]):sum(counts[:r + 1])] if grown[r] == counts[r] else None for r in range(self.n)]

    def commit(self, paths):
        """Keeps the nodes paths[r] of the step's trees, in their order."""
        path = torch.zeros(self.n, max(1, max(map(len, paths))), dtype=torch.int32)
        for r, p in enumerate(paths):
            path[r, :len(p)] = torch.tensor(p, dtype=torch.int32)
        accepted = torch.tensor([len(p) for p in paths], dtype=torch.int32, device=DEV)
        lens = torch.empty_like(self.lens)
        sg.colored_kv_commit(self.ctx, self.cache, self.table, self.lens, path.to(DEV), accepted, lens,
                             totals=self.totals)
        self.lens = lens

    def end(self):
        """Ends all requests; the pages that are free then."""
        totals, _, _ = self.map([-1] * self.n, 0)
        self.lens = totals
        taken, put = self.ring_pos.tolist()
        return put - taken


def draft(seq, depth):
    """A tree after the sequence's last token: the chain of what followed each
    token the last time, and what followed the last token the time before."""
    after = {}
    for a, b in zip(seq, seq[1:]):
        after.setdefault(a, []).append(b)
    tokens, parents = [seq[-1]], [-1]
    while len(tokens) <= depth and tokens[-1] in after:
        tokens.append(after[tokens[-1]][-1])
        parents.append(len(tokens) - 2)
    others = [t for t in after.get(seq[-1], []) if len(tokens) > 1 and t != tokens[1]]
    if others:
        tokens.append(others[-1])
        parents.append(0)
    return tokens, parents


def walk(tree, best):
    """The path that the model's own choices take through the tree, and the
    tokens that it gives: those of the path below the root and the next one."""
    tokens, parents = tree
    path = [0]
    while True:
        child = [i for i in range(path[-1] + 1, len(tokens)) if parents[i] == path[-1] and tokens[i] == best[path[-1]]]
        if not child:
            return path, [tokens[i] for i in path[1:]] + [best[path[-1]]]
        path.append(child[0])


def decode(ctx, weights, prompts, n_new, depth, blocks=None, counts=None):
    """n_new tokens or a few more after each prompt, and the steps they took, with
    ``blocks`` pages for all requests (None: as many as they can need).
    ``counts``: a dict that receives how many drafted nodes were accepted,
    tokens moved in the cache and requests not served, over all steps."""
    server = Server(ctx, weights, len(prompts), max(map(len, prompts)) + n_new + 2 * depth + 2 + BLOCK, blocks)
    seqs = [list(p) for p in prompts]
    trees = [(p, list(range(-1, len(p) - 1))) for p in prompts]   # chains
    steps, ended, seen = 0, 0, {"accepted": 0, "moved": 0, "not served": 0}
    while True:
        best = server.step(trees)
        paths = []
        for s, p, t, b in zip(seqs, prompts, trees, best):
            path, more = [], []
            if t is None or b is None:
                seen["not served"] += t is not None
            elif len(s) == len(p):
                path, more = list(range(len(p))), b[-1:]
            else:
                path, more = walk(t, b)
                seen["accepted"] += len(path) - 1
                seen["moved"] += sum(i != j for i, j in enumerate(path))
            paths.append(path)
            s += more
        server.commit(paths)
        steps += 1
        # no page becomes free, and no smaller draft is left to try
        if not any(paths) and trees.count(None) == ended and all(
                t is None or len(t[0]) == 1 or len(s) == len(p) for t, s, p in zip(trees, seqs, prompts)):
            raise RuntimeError("too few pages for any request to go on")
        ended = trees.count(None)
        if min(len(s) - len(p) for s, p in zip(seqs, prompts)) >= n_new:
            break
        # where the draft found no pages, the last token alone is next
        trees = [None if len(s) - len(p) >= n_new else (p, list(range(-1, len(p) - 1))) if len(s) == len(p) else
                 draft(s, 0 if b is None else depth) for s, p, b in zip(seqs, prompts, best)]
    free = server.end()
    assert free == server.ring.numel(), "a page was lost"
    assert ctx.device_error() == 0
    if counts is not None:
        counts.update(seen)
    return [s[len(p):len(p) + n_new] for s, p in zip(seqs, prompts)], steps


def main(n_new=48, depth=6, seed=3):
    ctx = sg.Context(0)
    try:
        weights = Weights(ctx, seed)
        g = torch.Generator().manual_seed(seed + 1)
        prompts = [torch.randint(0, VOCAB, (n,), generator=g).tolist() for n in (5, 37, 130)]
        alone, steps = decode(ctx, weights, prompts, n_new, 0)
        drafted, fewer = decode(ctx, weights, prompts, n_new, depth)
        same = sum(a == b for x, y in zip(alone, drafted) for a, b in zip(x, y))
        print(f"{len(prompts)} requests, {n_new} tokens each: {steps} steps one token at a time, {fewer} with "
              f"drafts; {same} of {n_new * len(prompts)} tokens agree")
        return weights, prompts, alone, drafted, steps, fewer
    finally:
        ctx.close()


if __name__ == "__main__":
    main()
