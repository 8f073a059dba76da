"""4-bit products, rotated writes and draft verification from four host threads at once, each on a stream of its own
with its own CUs; and caches and rows past 4 GiB."""
import threading

import pytest

import kv_oracle as ko
import paper_2407_13996_amd as sg
import test_gpu_draft_verify as tv
import test_gpu_kv_rotate as tr
import test_gpu_q4 as tq

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = sg.Context(0)
    yield c
    c.close()


class Work:
    """One thread's calls and what they gave alone."""

    def __init__(self, ctx, i):
        self.m = tq.Matrix(1500 + 700 * i, 1152, 64, sg.BF16, i % 2 == 1, 12, seed=i).upload(ctx)
        self.x = tq.inputs(self.m, 1 + 5 * i, seed=i).to(DEV)
        self.c = tr.Call(200 + 90 * i, 8, 2, 128, 32, sg.BF16, 128, False, "qk", seed=i)
        self.q = [t.to(DEV) for t in (self.c.proj, self.c.slots, self.c.position, self.c.freq, self.c.q_norm,
                                      self.c.k_norm)]
        self.pool = self.c.pool.to(DEV)
        self.v = [t.to(DEV) for t in tv.case([3 + i, 6], 100003, "tree", "f32", 50 + i)]
        torch.cuda.synchronize()
        self.want = self.run(ctx, None)
        torch.cuda.synchronize()

    def run(self, ctx, stream):
        y = torch.full((self.x.shape[0], self.m.q.rows), -1.0, device=DEV)
        sg.colored_gemv_q4(ctx, self.m.w, self.m.q, self.x, self.x.shape[0], y, self.m.shift, stream=stream)
        pool, (proj, slots, position, freq, qn, kn) = self.pool.clone(), self.q
        q, k, v = self.c.parts(proj)
        out = torch.zeros(q.shape, dtype=q.dtype, device=DEV)
        cache = sg.kv_cache(pool, self.c.pages, self.c.shift, 32, 2, 128, sg.BF16)
        sg.colored_kv_append_rotated(ctx, cache, 0, q, k, v, out, slots, position, freq=freq, q_norm=qn, k_norm=kn,
                                     eps=1e-5, stream=stream)
        target, guess, tokens, parents, u, q_start = self.v
        path = torch.zeros(2, 16, dtype=torch.int32, device=DEV)
        accepted, after = (torch.zeros(2, dtype=torch.int32, device=DEV) for _ in range(2))
        sg.colored_draft_verify(ctx, target, tokens, parents, u, q_start, path, accepted, after, draft=guess,
                                stream=stream)
        return y, pool, out, path, accepted, after


def test_threads(ctx):
    works = [Work(ctx, i) for i in range(4)]
    assert ctx.device_error() == 0
    failed = []

    def go(i):
        try:
            s = torch.cuda.Stream()
            sg.set_cu_mask(ctx, s, [None, range(64, 128), range(7, 90), [3, 150, 200]][i])
            with torch.cuda.stream(s):
                for n in range(12):
                    got = works[i].run(ctx, s)
                    s.synchronize()
                    for k, (a, b) in enumerate(zip(got, works[i].want)):
                        if not torch.equal(a.view(torch.uint8), b.view(torch.uint8)):
                            failed.append((i, n, k))
            sg.stream_release(ctx, s)
        except Exception as e:  # noqa: BLE001
            failed.append((i, repr(e)))

    threads = [threading.Thread(target=go, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
    assert ctx.device_error() == 0


def test_rotated_writes_past_4_gib(ctx):
    """Pages whose addresses pass 32 bits, and rows of q and q_out past 2^32 bytes, at the
    widest stride that rows may have."""
    n, heads, kv, dim, block = 4, 4, 2, 128, 16
    elems, shift = ko.pages_of(kv, dim, block, 1)
    pages = (5 << 30) >> shift
    pool = torch.zeros(pages << (shift - 1), dtype=torch.int16, device=DEV)
    g = torch.Generator().manual_seed(1)
    proj = torch.randn(n, heads + 2 * kv, dim, generator=g).to(torch.bfloat16)
    apart = 1 << 30                                        # elements from a token to the next
    wide = torch.zeros((n - 1) * apart + (heads + 2 * kv) * dim, dtype=torch.bfloat16, device=DEV)
    rows = wide.as_strided((n, heads + 2 * kv, dim), (apart, dim, 1))
    rows.copy_(proj)
    q, k, v = rows[:, :heads], rows[:, heads:heads + kv], rows[:, heads + kv:]
    slots = torch.tensor([5, pages * block - 1, (pages - 2) * block + 3, 100])
    position = torch.tensor([7, 123456, 2 ** 31 - 1, 0], dtype=torch.int32)
    freq = tr.angles(dim // 2)
    cache = sg.kv_cache(pool, pages, shift, block, kv, dim, sg.BF16)
    sg.colored_kv_append_rotated(ctx, cache, 0, q, k, v, q, slots.to(DEV), position.to(DEV), freq=freq.to(DEV))
    torch.cuda.synchronize()
    assert ctx.device_error() == 0
    want, err = tr.turned(proj[:, :heads], position, freq, None, 0.0, False)
    tr.close(q.cpu(), want, err, torch.bfloat16)
    per = 1 << (shift - 1)
    for t, s in enumerate(slots.tolist()):
        page = pool[(s // block) * per:(s // block + 1) * per].cpu()
        at = torch.tensor([s % block])
        got = ko.rows(page, ko.k_index, per, block, kv, dim, at).contiguous().view(torch.bfloat16)
        want, err = tr.turned(proj[t:t + 1, heads:heads + kv], position[t:t + 1], freq, None, 0.0, False)
        tr.close(got, want, err, torch.bfloat16)
        got = ko.rows(page, ko.v_index, per, block, kv, dim, at).contiguous().view(torch.bfloat16)
        assert torch.equal(got, proj[t:t + 1, heads + kv:])
    assert int((pool != 0).sum()) <= n * 2 * kv * dim
