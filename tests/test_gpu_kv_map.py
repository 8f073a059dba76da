"""Block tables and slot maps built on the GPU, against request-after-request
loops on the host: every output equal, over steps of a server's life (pages
taken from and returned to a ring that wraps around), odd sizes, shortfalls
and states out of range."""
import numpy as np
import pytest

import kv_oracle as ko
import paper_2407_13996_amd as sg

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = sg.Context(0)
    yield c
    c.close()


def dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype=dtype))).to(DEV)


def step(ctx, block, st, new, n_tokens):
    """One call and its oracle on copies of the state; returns both."""
    r = len(new)
    d = {k: dev(st[k], np.int64 if k == "ring_pos" else np.int32) for k in ("ring_pos", "held", "lens", "ring")}
    table, out = dev(st["table"]), {}
    for k, n, t in (("ring_pos", 2, torch.int64), ("held", r, torch.int32), ("lens", r, torch.int32),
                    ("q_start", r + 1, torch.int32), ("slots", n_tokens, torch.int64),
                    ("request", n_tokens, torch.int32), ("position", n_tokens, torch.int32)):
        out[k] = torch.full((n,), -77, dtype=t, device=DEV)
    sg.colored_kv_map(ctx, block, d["ring"], d["ring_pos"], d["held"], d["lens"], dev(new), table, out["ring_pos"],
                      out["held"], out["lens"], out["q_start"], out["slots"], out["request"], out["position"])
    torch.cuda.synchronize()
    flags = ctx.device_error()
    got = {k: v.cpu().numpy() for k, v in out.items()}
    got["table"], got["ring"] = table.cpu().numpy(), d["ring"].cpu().numpy()
    want_table, want_ring = np.array(st["table"]), np.array(st["ring"])
    want = ko.kv_map(block, want_ring, st["ring_pos"], np.asarray(st["held"]), np.asarray(st["lens"]),
                     np.asarray(new), want_table, n_tokens)
    want["table"], want["ring"] = want_table, want_ring
    assert bool(flags & sg.DEVERR_SEQ) == want.pop("flag"), flags
    for k, w in want.items():
        assert np.array_equal(got[k], np.asarray(w)), k
    return want


def start(requests, width, pages, seed, taken=0):
    rng = np.random.default_rng(seed)
    return {"ring": rng.permutation(pages).astype(np.int32), "ring_pos": [taken, taken + pages],
            "held": np.zeros(requests, int), "lens": np.zeros(requests, int),
            "table": np.full((requests, width), -1, np.int32)}, rng


@pytest.mark.parametrize("requests,block,most,pages", [(1, 16, 1, 40), (3, 16, 40, 30), (64, 32, 5, 300),
                                                        (257, 16, 9, 700), (1030, 64, 70, 2500), (4096, 16, 3, 9000)])
def test_steps_of_a_server(ctx, requests, block, most, pages):
    """Six steps: requests grow, some end, and the ring runs short and recovers."""
    st, rng = start(requests, 12, pages, requests, taken=(1 << 33) + 5)
    for _ in range(6):
        room = 12 * block - st["lens"]
        new = np.minimum(rng.integers(0, most + 1, requests), np.maximum(room, 0))
        new = np.where(rng.random(requests) < 0.15, -1, new)
        tokens = int(np.maximum(new, 0).sum())
        w = step(ctx, block, st, new, tokens + int(rng.integers(0, 3)))
        st = {"ring": w["ring"], "ring_pos": w["ring_pos"], "held": np.array(w["held"]), "lens": np.array(w["lens"]),
              "table": w["table"]}


def test_a_shortfall_serves_those_before_it_and_those_that_need_nothing(ctx):
    st, _ = start(5, 4, 8, 0)
    st.update(ring_pos=[0, 3], held=np.array([1, 1, 1, 1, 1]), lens=np.array([16, 15, 16, 3, 16]))
    st["table"][:, 0] = [100, 101, 102, 103, 104]
    w = step(ctx, 16, st, np.array([17, 1, 33, 2, 0]), 60)
    assert w["lens"] == [33, 16, 16, 5, 16] and w["ring_pos"][0] == 2


def test_long_prompts_fill_whole_rows(ctx):
    st, _ = start(2, 700, 1500, 3)
    w = step(ctx, 16, st, np.array([700 * 16, 5001]), 700 * 16 + 5001)
    assert w["held"] == [700, 313]


def test_states_out_of_range_are_refused_and_flagged(ctx):
    # lengths that no row holds, negative ones, more blocks than a row, a row that overflows
    st, _ = start(8, 4, 64, 1)
    st.update(held=np.array([4, 1, 5, -1, 2, 0, 1, 1]), lens=np.array([65, -3, 20, 0, 20, 1, 16, 9]))
    st["table"][:] = np.arange(32).reshape(8, 4)
    step(ctx, 16, st, np.array([1, 1, 1, 1, 45, 1, 2, -1]), 60)
    st["held"], st["lens"] = np.array([1] * 8), np.array([16] * 8)
    step(ctx, 16, st, np.array([1] * 8), 8)                       # sound again: no flag
    st["ring_pos"] = [10, 5]                                      # a ring that gave more than it had
    step(ctx, 16, st, np.array([1, 0, -1, 1, 0, 0, 0, 0]), 8)
    st["ring_pos"] = [0, 1000]                                    # or holds more than fit
    step(ctx, 16, st, np.array([1, 0, 1, 1, 0, 0, 0, 0]), 8)


def test_tokens_past_the_arrays_are_refused(ctx):
    st, _ = start(4, 4, 64, 2)
    step(ctx, 16, st, np.array([5, 6, 7, 0]), 12)
    step(ctx, 16, st, np.array([5, 6, 7, 0]), 11)
    step(ctx, 16, st, np.array([0, 0, 0, 0]), 0)
    step(ctx, 16, st, np.array([3, 0, -1, 0]), 0)
    step(ctx, 16, st, np.array([2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 4]), 30)


@pytest.mark.parametrize("cus", [list(range(64)), [3, 40, 41, 77, 130, 255]])
def test_any_cu_mask_gives_the_same(ctx, cus):
    sg.set_cu_mask(ctx, None, cus)
    try:
        st, rng = start(500, 8, 3000, 9)
        step(ctx, 32, st, rng.integers(0, 60, 500), 30000)
    finally:
        sg.set_cu_mask(ctx, None, None)


def test_bindings_refuse_arrays_that_do_not_fit(ctx):
    z = lambda n, t=torch.int32: torch.zeros(n, dtype=t, device=DEV)  # noqa: E731
    a = dict(ring=z(8), ring_pos=z(2, torch.int64), held=z(3), lens=z(3), new=z(3), table=z(12).view(3, 4),
             ring_pos_out=z(2, torch.int64), held_out=z(3), lens_out=z(3), q_start=z(4), slots=z(5, torch.int64),
             request=z(5), position=z(5))
    for name, bad in (("held", z(2)), ("q_start", z(3)), ("request", z(4)), ("slots", z(5)), ("lens", z(6)[::2]),
                      ("ring_pos", z(2)), ("table", z(12).view(4, 3).t()), ("new", torch.zeros(3, device=DEV))):
        with pytest.raises(ValueError):
            sg.colored_kv_map(ctx, 16, **{**a, name: bad})
    with pytest.raises(sg.SgdrcError):
        sg.colored_kv_map(ctx, 16, **{**a, "held_out": a["held"]})
    with pytest.raises(sg.SgdrcError):
        sg.colored_kv_map(ctx, 17, **a)
