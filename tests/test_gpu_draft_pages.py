"""Decoding with drafts: that drafts are accepted, side branches among them, and
that requests wait where the pages do not reach for all."""
import pytest

import paper_2407_13996_amd as sg
from test_gpu_draft_decoding import logits_of

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
N_NEW = 48


@pytest.fixture(scope="module")
def model():
    import draft_decoding as dd
    ctx = sg.Context(0)
    yield dd, ctx, dd.Weights(ctx, 3)
    ctx.close()


def check(dd, weights, prompts, new):
    """Every token is the model's own choice, up to the roundings of two layers
    and the last norm (as in test_drafts_give_the_models_tokens)."""
    for p, n in zip(prompts, new):
        assert len(n) == N_NEW
        rows = logits_of(dd, weights, p + n)[len(p) - 1:-1]
        got = rows.gather(1, torch.tensor(n)[:, None])[:, 0]
        assert bool((got >= rows.max(1).values - 32 * 2.0 ** -9).all())


def prompts_of(lengths, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randint(0, 384, (n,), generator=g).tolist() for n in lengths]


def test_side_branches_are_accepted_and_closed_up(model, monkeypatch):
    """Drafts whose first guess is wrong and whose side branch is what the model said
    without drafts, two tokens deep: both move in the cache."""
    dd, ctx, weights = model
    prompts = prompts_of((5, 37, 130), 4)
    alone, steps = dd.decode(ctx, weights, prompts, N_NEW, 0)
    assert steps == N_NEW

    def draft(seq, depth):
        p, said = next((p, n) for p, n in zip(prompts, alone) if seq[:len(p)] == p)
        right = (said + [0, 0])[len(seq) - len(p):][:2]
        return [seq[-1], (right[0] + 1) % dd.VOCAB] + right, [-1, 0, 0, 2]

    monkeypatch.setattr(dd, "draft", draft)
    counts = {}
    new, fewer = dd.decode(ctx, weights, prompts, N_NEW, 3, counts=counts)
    check(dd, weights, prompts, new)
    assert counts["not served"] == 0
    # nearly all: where two tokens are as good, drafts may take another than the one before
    assert counts["moved"] == counts["accepted"] >= N_NEW and fewer <= N_NEW // 2


@pytest.mark.parametrize("depth", [0, 6])
def test_requests_wait_for_pages(model, depth):
    """Twelve pages of 16 tokens: the prompt of 130 begins once the others have ended."""
    dd, ctx, weights = model
    prompts = prompts_of((5, 37, 130), 4)
    counts = {}
    new, steps = dd.decode(ctx, weights, prompts, N_NEW, depth, blocks=12, counts=counts)
    check(dd, weights, prompts, new)
    assert counts["not served"] > 0 and steps > N_NEW // 2


def test_too_few_pages_for_anything(model):
    dd, ctx, weights = model
    for lengths in ((40,), (5, 130)):      # the second has pages only without the first, and then not enough
        with pytest.raises(RuntimeError):
            dd.decode(ctx, weights, prompts_of(lengths, 1), N_NEW, 0, blocks=2 if len(lengths) == 1 else 6)
    ctx.device_error()


def test_a_draft_that_does_not_fit_gives_way_to_its_root(model, monkeypatch):
    """One request whose drafts of 40 nodes never find the pages that its tokens do."""
    dd, ctx, weights = model
    prompts = prompts_of((20,), 2)
    monkeypatch.setattr(dd, "draft", lambda seq, depth: (seq[-1:] + [1] * 39 * (depth > 0),
                                                         list(range(-1, 39 if depth else 0))))
    counts = {}
    new, _ = dd.decode(ctx, weights, prompts, N_NEW, 6, blocks=5, counts=counts)
    check(dd, weights, prompts, new)
    assert counts["not served"] > 0
