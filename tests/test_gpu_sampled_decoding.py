"""4-bit products, rotated writes, attention, verification and commits in one serving loop: the
logits against the same model in 64 bits without a cache, each step's accepted path and
token against the verification in 64 bits on the probabilities that the step had."""
import os
import sys

import pytest

import verify_oracle as vo

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def logits_of(sd, w, seq):
    """The model's logits after every token of a sequence, in 64 bits."""
    f, dd = torch.float64, sd.dd
    plain = {n: t.cpu().to(f) for n, t in w.plain.items()}
    x, n, group = w.embed.cpu().to(f)[seq], len(seq), sd.HEADS // sd.KV
    angle = torch.arange(n, dtype=f)[:, None, None] * w.freq.cpu().to(f)

    def turn(t, weight):
        t = t / torch.sqrt(t.square().mean(-1, keepdim=True) + sd.EPS) * weight.cpu().to(f)
        a, b = t.chunk(2, -1)
        return torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1)

    for layer in range(sd.LAYERS):
        qkv = (dd.norm(x) @ plain[f"qkv{layer}"].T).view(n, sd.HEADS + 2 * sd.KV, sd.DIM)
        q, k, v = qkv.split([sd.HEADS, sd.KV, sd.KV], 1)
        q, k = turn(q, w.norms[layer][0]), turn(k, w.norms[layer][1])
        s = torch.einsum("ihd,jhd->hij", q, k.repeat_interleave(group, 1)) * sd.DIM ** -0.5
        s = s.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -torch.inf)
        o = torch.einsum("hij,jhd->ihd", s.softmax(-1), v.repeat_interleave(group, 1))
        x = x + o.reshape(n, -1) @ plain[f"out{layer}"].T
    return dd.norm(x) @ plain["logits"].T


def test_the_samples_are_the_models():
    import sampled_decoding as sd
    seen = []
    w, prompts, seqs, steps = sd.main(n_new=40, depth=4, width=3, seen=seen)
    assert steps == len(seen) + 1
    whole = [logits_of(sd, w, s) for s in seqs]
    # A layer rounds its input, the projections, q and k once more when turned, the softmax's weights
    # and its result to 8 bits, 2^-8 of their size each (half a step); two layers and the last
    # norm are some ten in a row, of which each moves the logits by that part of their size.
    tol = 10 * 2.0 ** -8
    at = [len(p) for p in prompts]          # of each request's root
    most = 0
    for logits, target, draft, tokens, parents, uniform, q_start, lens, totals, path, accepted, after in seen:
        f = lambda t: t.cpu().double().numpy()  # noqa: E731
        i = lambda t: t.cpu().numpy()  # noqa: E731
        paths, counts, nxt, flag = vo.verify(f(target), f(draft), i(tokens), i(parents), f(uniform), i(q_start),
                                             path.shape[1], 256, lens=i(lens), totals=i(totals))
        assert (path.tolist(), accepted.tolist(), after.tolist(), flag) == (paths, counts, nxt, False)
        start = q_start.tolist()
        for r, n in enumerate(counts):
            if start[r] == start[r + 1]:
                continue
            assert lens[r] == at[r]
            nodes = [start[r] + k for k in paths[r][:n]]
            assert tokens[nodes].tolist() == seqs[r][at[r]:at[r] + n]
            want = whole[r][at[r]:at[r] + n]
            off = (logits[nodes].cpu().double() - want).abs().max(1).values / want.abs().max(1).values
            assert bool((off <= tol).all()), off
            most, at[r] = max(most, n), at[r] + n
    assert at == [len(s) - 1 for s in seqs]
    assert most > 1                         # drafts were accepted


def test_trees_are_drawn_from_their_parents():
    import sampled_decoding as sd
    guess = torch.roll(torch.eye(7), 1, 1)  # after t comes t + 1
    g = torch.Generator().manual_seed(0)
    assert sd.draw_tree(guess, 2, 4, 3, g) == ([2, 3, 3, 3, 4, 5, 6], [-1, 0, 0, 0, 1, 4, 5])
    assert sd.draw_tree(guess, 6, 1, 1, g) == ([6, 0], [-1, 0])
