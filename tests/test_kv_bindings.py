"""What the cache's bindings make of tensors before anything is called: no GPU needed."""
import pytest

import paper_2407_13996_amd as sg

torch = pytest.importorskip("torch")


def test_strides_that_nothing_uses_are_not_refused():
    """One token of a projection whose rows are no multiple of 8 long; one head of such a one."""
    proj = torch.zeros(3, 4 * 64 + 4, dtype=torch.float16)
    one = proj.as_strided((1, 4, 64), (260, 64, 1))
    assert one.stride(0) % 8
    r = sg._rows(one, "q", 4, 64, sg.F16)
    assert (r.ptr, r.token_stride, r.head_stride) == (proj.data_ptr(), 0, 64)
    head = torch.zeros(5, 3, 68, dtype=torch.float16).as_strided((5, 1, 64), (204, 68, 1))
    assert sg._rows(head, "q", 1, 64, sg.F16).head_stride == 0
    both = torch.zeros(5, 3, 64, dtype=torch.float16)
    r = sg._rows(both, "q", 3, 64, sg.F16)
    assert (r.token_stride, r.head_stride) == (192, 64)


def aligned(n):
    """n bytes from a multiple of 256 on."""
    t = torch.zeros(n + 256, dtype=torch.uint8)
    return t[-t.data_ptr() % 256:][:n]


def attend(**kw):
    cache = sg.kv_cache(aligned(1 << 12), 1, 12, 16, 1, 64, sg.F16)
    a = dict(q=torch.zeros(3, 2, 64, dtype=torch.float16), q_start=torch.zeros(2, dtype=torch.int32),
             table=torch.zeros(1, 1, dtype=torch.int32), lens=torch.zeros(1, dtype=torch.int32),
             totals=torch.zeros(1, dtype=torch.int32), out=torch.zeros(3, 2, 64, dtype=torch.float16),
             work=aligned(1 << 23), max_nodes=3, stream=0)
    a.update(kw)
    sg.colored_tree_attention(None, cache, 0, **a)


def test_results_and_workspaces_that_share_memory_are_refused():
    """Sound ones get as far as the missing context."""
    half = torch.zeros(3, 2, 64, dtype=torch.float16)
    pairs = torch.zeros(2, 3, 64, dtype=torch.float16).transpose(0, 1)         # heads outside, tokens inside
    wide = torch.zeros(3, 5, 64, dtype=torch.float16)[:, 1:3]
    for out in (half, pairs, wide):
        with pytest.raises(sg.SgdrcError) as e:
            attend(out=out)
        assert e.value.code == sg.ENODEV
    for out in (half[:1].expand(3, 2, 64), half[:, :1].expand(3, 2, 64),
                torch.zeros(400, dtype=torch.float16).as_strided((3, 2, 64), (64, 64, 1)),
                torch.zeros(400, dtype=torch.float16).as_strided((3, 2, 64), (128, 32, 1))):
        with pytest.raises(ValueError):
            attend(out=out)
    for work in (torch.zeros(1, dtype=torch.uint8).expand(1 << 23), aligned(1 << 24)[::2], 4096):
        with pytest.raises(ValueError):
            attend(work=work)
