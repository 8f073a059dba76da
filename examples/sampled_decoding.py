"""Sampling with drafted trees from a decoder with 4-bit weights.

The serving loop of draft_decoding.py (prompts as chains, pages of chosen
colours, trees of drafted tokens) for a decoder as they are served mostly: its
projections lie in the pool as 4-bit weights with group scales and zero points
(colored_q4_pack, colored_gemv_q4), queries and keys have norms and a rotation
by their position, applied on the way into the cache (colored_kv_append_rotated), and
the tokens are sampled: each step draws a tree from a small model's distribution
-- here the big model without its layers, a table -- and colored_draft_verify accepts
of it what keeps the big model's own distribution.  Its path and counts go to
colored_kv_commit on the device.  Run on an MI355X:

    python examples/sampled_decoding.py
"""
import torch

import draft_decoding as dd
import paper_2407_13996_amd as sg
from draft_decoding import BLOCK, DEV, DIM, HEADS, HIDDEN, KV, LAYERS, MOST, SHIFT, VOCAB

GROUP = 64                            # columns of a scale
EPS = 1e-6


def quantise(w):
    """Codes (0..15), scales and zero points of a matrix, and the matrix that they mean."""
    parts = w.float().view(w.shape[0], -1, GROUP)
    low, high = parts.amin(-1).clamp(max=0), parts.amax(-1).clamp(min=0)
    scales = ((high - low) / 15).clamp(min=1e-8).to(torch.bfloat16)
    zeros = (-low / scales.float()).round().clamp(0, 15).to(torch.bfloat16)
    s, z = scales.float()[..., None], zeros.float()[..., None]
    codes = (parts / s + z).round().clamp(0, 15)
    return codes.to(torch.uint8).view(w.shape), scales, zeros, (s * (codes - z)).view(w.shape)


class Weights:
    """Random weights; all matrices but the last one in 4 bits."""

    def __init__(self, ctx, seed):
        g = torch.Generator().manual_seed(seed)

        def normal(*shape, scale=1.0):
            return (torch.randn(*shape, generator=g) * scale).to(torch.bfloat16).to(DEV)

        self.embed, self.plain, self.paged, self.q4, self.norms = normal(VOCAB, HIDDEN), {}, {}, {}, {}
        for layer in range(LAYERS):
            for name, rows, cols in (("qkv", (HEADS + 2 * KV) * DIM, HIDDEN), ("out", HIDDEN, HEADS * DIM)):
                codes, scales, zeros, self.plain[f"{name}{layer}"] = quantise(normal(rows, cols, scale=cols ** -0.5))
                q = sg.q4(rows, cols, GROUP, sg.BF16, zeros=True)
                pool, table, pages = dd.coloured_pages(ctx, -(-sg.q4_bytes(q) >> SHIFT))
                w = sg.paged(pool, table, pages)
                sg.colored_q4_pack(ctx, w, q, codes, scales, zeros, SHIFT)
                self.q4[f"{name}{layer}"], self.paged[f"{name}{layer}"] = q, w
            self.norms[layer] = [1 + normal(DIM, scale=0.1) for _ in range(2)]
        self.plain["logits"] = normal(VOCAB, HIDDEN, scale=2 * HIDDEN ** -0.5)
        self.paged["logits"] = dd.coloured_copy(ctx, self.plain["logits"])
        self.freq = 10000.0 ** (-torch.arange(DIM // 2, device=DEV) / (DIM // 2))

    def apply(self, ctx, name, x):
        """x @ W^T in fp32: 4-bit matrices sixteen tokens a call, bf16 ones eight."""
        rows, k = self.plain[name].shape
        x = x.to(torch.bfloat16).contiguous()
        y = torch.empty(x.shape[0], rows, dtype=torch.float32, device=DEV)
        most = 16 if name in self.q4 else 8
        for t in range(0, x.shape[0], most):
            n = min(most, x.shape[0] - t)
            if name in self.q4:
                sg.colored_gemv_q4(ctx, self.paged[name], self.q4[name], x[t:t + n], n, y[t:t + n], SHIFT)
            else:
                sg.colored_gemv(ctx, self.paged[name], sg.BF16, rows, k, x[t:], sg.BF16, n, y[t:], SHIFT)
        return y


class Server(dd.Server):
    def step(self, trees):
        """Logits after every node of the requests' trees (tokens, parents;
        None: the request ends), and where each request's nodes begin."""
        new = [-1 if t is None else len(t[0]) for t in trees]
        trees = [t or ([], []) for t in trees]
        counts = [len(t) for t, _ in trees]
        n = sum(counts)
        tokens = torch.tensor([t for tree, _ in trees for t in tree], device=DEV)
        mask, depth = dd.masks_and_depths(trees)
        self.totals, q_start, slots = self.map(new, n)
        at = self.lens.repeat_interleave(torch.tensor(counts, device=DEV)) + torch.tensor(depth, dtype=torch.int32,
                                                                                         device=DEV)
        x = self.w.embed[tokens].float()
        for layer in range(LAYERS):
            qkv = self.w.apply(self.ctx, f"qkv{layer}", dd.norm(x)).to(torch.bfloat16).view(n, HEADS + 2 * KV, DIM)
            q, k, v = qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV], qkv[:, HEADS + KV:]
            q_norm, k_norm = self.w.norms[layer]
            sg.colored_kv_append_rotated(self.ctx, self.cache, layer, q, k, v, q, slots, at, freq=self.w.freq,
                                         q_norm=q_norm, k_norm=k_norm, eps=EPS)
            o = torch.empty(n, HEADS, DIM, dtype=torch.bfloat16, device=DEV)
            sg.colored_tree_attention(self.ctx, self.cache, layer, q, q_start, self.table, self.lens, self.totals, o,
                                      self.work, mask=mask, max_nodes=MOST, scale=DIM ** -0.5)
            x = x + self.w.apply(self.ctx, f"out{layer}", o.view(n, HEADS * DIM))
        return self.w.apply(self.ctx, "logits", dd.norm(x)), q_start

    def verify(self, tokens, parents, target, draft, uniform, q_start, most):
        """Accepts of the step's trees what a sampler of ``target`` would, and keeps it in the cache."""
        path = torch.empty(self.n, most, dtype=torch.int32, device=DEV)
        accepted, after, lens = (torch.empty(self.n, dtype=torch.int32, device=DEV) for _ in range(3))
        sg.colored_draft_verify(self.ctx, target, tokens, parents, uniform, q_start, path, accepted, after,
                                draft=draft, lens=self.lens, totals=self.totals)
        sg.colored_kv_commit(self.ctx, self.cache, self.table, self.lens, path, accepted, lens, totals=self.totals)
        self.lens = lens
        return path, accepted, after


def draw_tree(guess, last, depth, width, g):
    """``width`` children of the last token and a chain below the first, each token
    drawn from its parent's row of ``guess``."""
    tokens, parents = [last], [-1]
    for _ in range(width):
        tokens.append(int(torch.multinomial(guess[last], 1, generator=g)))
        parents.append(0)
    for i in range(1, depth):
        tokens.append(int(torch.multinomial(guess[tokens[1 if i == 1 else -1]], 1, generator=g)))
        parents.append(1 if i == 1 else len(tokens) - 2)
    return tokens, parents


def decode(ctx, weights, prompts, n_new, depth, width, seed, temperature=1.0, seen=None):
    """n_new sampled tokens or a few more after each prompt, and the steps they took.
    ``seen``: a list that receives the steps' (logits, target, draft, tokens,
    parents, uniform, q_start, lens, totals, path, accepted, next)."""
    g = torch.Generator().manual_seed(seed)
    nodes = 1 + width + max(0, depth - 1)
    server = Server(ctx, weights, len(prompts), max(map(len, prompts)) + n_new + 2 * nodes + BLOCK)
    # the small model: what a token alone says
    guess = torch.softmax(weights.apply(ctx, "logits", dd.norm(weights.embed.float())) / temperature, 1)
    table = guess.cpu()
    seqs = [list(p) for p in prompts]
    logits, q_start = server.step([(p, list(range(-1, len(p) - 1))) for p in prompts])
    # a prompt's first token: a tree of one node, after the last of the prompt
    rows, n = q_start[1:].long() - 1, len(prompts)
    target = torch.softmax(logits[rows] / temperature, 1)
    firsts = torch.arange(n + 1, dtype=torch.int32, device=DEV)
    roots = torch.tensor([p[-1] for p in prompts], dtype=torch.int32, device=DEV)
    path, accepted, after = (torch.empty(n, *w, dtype=torch.int32, device=DEV) for w in ((1,), (), ()))
    sg.colored_draft_verify(ctx, target, roots, torch.full_like(roots, -1), torch.rand(n, generator=g).to(DEV), firsts,
                            path, accepted, after)
    server.commit([list(range(len(p))) for p in prompts])
    for s, t in zip(seqs, after.tolist()):
        s.append(t)
    steps = 1
    while min(len(s) - len(p) for s, p in zip(seqs, prompts)) < n_new:
        trees = [draw_tree(table, s[-1], depth, width, g) if len(s) - len(p) < n_new else None
                 for s, p in zip(seqs, prompts)]
        tokens, parents = (torch.tensor([x for t in trees if t for x in t[i]], dtype=torch.int32, device=DEV)
                           for i in (0, 1))
        lens = server.lens
        logits, q_start = server.step(trees)
        target = torch.softmax(logits / temperature, 1)
        draft, uniform = guess[tokens.long()], torch.rand(tokens.numel(), generator=g).to(DEV)
        path, accepted, after = server.verify(tokens, parents, target, draft, uniform, q_start, depth + 1)
        if seen is not None:
            seen.append((logits, target, draft, tokens, parents, uniform, q_start, lens, server.totals, path, accepted,
                         after))
        for s, t, p, a, x in zip(seqs, trees, path.tolist(), accepted.tolist(), after.tolist()):
            if t:
                s += [t[0][i] for i in p[1:a]] + [x]
        steps += 1
    free = server.end()
    assert free == server.ring.numel(), "a page was lost"
    assert ctx.device_error() == 0
    return seqs, steps


def main(n_new=48, depth=4, width=3, seed=3, seen=None):
    ctx = sg.Context(0)
    try:
        weights = Weights(ctx, seed)
        g = torch.Generator().manual_seed(seed + 1)
        prompts = [torch.randint(0, VOCAB, (n,), generator=g).tolist() for n in (5, 37, 130)]
        seqs, steps = decode(ctx, weights, prompts, n_new, depth, width, seed + 2, seen=seen)
        made = sum(len(s) - len(p) for s, p in zip(seqs, prompts))
        print(f"{len(prompts)} requests: {made} tokens sampled in {steps} steps")
        return weights, prompts, seqs, steps
    finally:
        ctx.close()


if __name__ == "__main__":
    main()
