"""Decoding with drafts, all the cache's operators together, against the same
model in 64 bits without a cache."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def logits_of(dd, w, seq):
    """The model's logits after every token of a sequence, in 64 bits."""
    f = torch.float64
    plain = {n: t.cpu().to(f) for n, t in w.plain.items()}
    x = w.embed.cpu().to(f)[seq] + w.place.cpu().to(f)[:len(seq)]
    n, group = len(seq), dd.HEADS // dd.KV
    for layer in range(dd.LAYERS):
        qkv = (dd.norm(x) @ plain[f"qkv{layer}"].T).view(n, dd.HEADS + 2 * dd.KV, dd.DIM)
        q, k, v = qkv.split([dd.HEADS, dd.KV, dd.KV], 1)
        s = torch.einsum("ihd,jhd->hij", q, k.repeat_interleave(group, 1)) * dd.DIM ** -0.5
        s = s.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -torch.inf)
        o = torch.einsum("hij,jhd->ihd", s.softmax(-1), v.repeat_interleave(group, 1))
        x = x + o.reshape(n, -1) @ plain[f"out{layer}"].T
    return dd.norm(x) @ plain["logits"].T


def test_drafts_give_the_models_tokens():
    import draft_decoding as dd
    w, prompts, alone, drafted, steps, fewer = dd.main(n_new=40, depth=5)
    assert fewer <= steps
    # A layer rounds its input, q, k, v, the weights of the softmax, its result
    # to 8 bits, 2^-9 each; two layers and the last norm keep that at some ten
    # such steps of the logits' size, which is about 1.
    tol = 32 * 2.0 ** -9
    for p, a, d in zip(prompts, alone, drafted):
        for new in (a, d):
            assert len(new) == 40
            rows = logits_of(dd, w, p + new)[len(p) - 1:-1]
            got = rows.gather(1, torch.tensor(new)[:, None])[:, 0]
            assert bool((got >= rows.max(1).values - tol).all()), float((rows.max(1).values - got).max())


def test_a_tree_is_walked_as_far_as_it_is_right():
    import draft_decoding as dd
    tree = dd.draft([1, 2, 3, 1, 4, 1, 2, 9, 1], 3)
    assert tree == ([1, 2, 9, 1, 4], [-1, 0, 1, 2, 0])
    assert dd.walk(tree, [2, 9, 1, 7, 0]) == ([0, 1, 2, 3], [2, 9, 1, 7])
    assert dd.walk(tree, [4, 0, 0, 0, 5]) == ([0, 4], [4, 5])
    assert dd.walk(tree, [8, 0, 0, 0, 0]) == ([0], [8])
