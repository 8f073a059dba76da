"""colored_kv_commit_within refuses what colored_kv_commit does, and totals that
are no lengths, on the host: no GPU needed."""
import ctypes

import pytest

import paper_2407_13996_amd as sg
from test_kv_abi import BAD_BLOCKS, BAD_CACHES, blocks, cache

r = ctypes.byref


def within(c=None, b=None, lens=256, totals=1024, path=256, stride=4, accepted=256, out=512):
    return sg.lib().colored_kv_commit_within(None, r(c or cache()), r(b or blocks()), lens, totals, path, stride,
                                             accepted, out, None)


def test_refusals():
    assert within() == within(totals=256) == sg.ENODEV
    for kw in (dict(lens=0), dict(totals=0), dict(totals=258), dict(totals=512), dict(path=0), dict(accepted=2),
               dict(out=0), dict(out=256), dict(stride=0), dict(stride=257)):
        assert within(**kw) == sg.EINVAL, kw
    for bad in BAD_CACHES:
        assert within(c=cache(**bad)) == sg.EINVAL, bad
    for bad in BAD_BLOCKS:
        assert within(b=blocks(**bad)) == sg.EINVAL, bad


def test_binding_refuses_totals_that_do_not_fit():
    torch = pytest.importorskip("torch")
    z = lambda *n: torch.zeros(*n, dtype=torch.int32)  # noqa: E731
    c = sg.kv_cache(z(64), 4, 12, 16, 1, 64, sg.F16)
    for bad in (z(2), z(4), z(3).long(), z(6)[::2], torch.zeros(3)):
        with pytest.raises(ValueError):
            sg.colored_kv_commit(None, c, z(3, 4), z(3), z(3, 2), z(3), z(3), stream=0, totals=bad)
