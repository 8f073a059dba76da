"""Block tables that are part of wider ones, on the host: the rows' width is
what the caller's view has, not how far its rows lie apart.  No GPU needed."""
import ctypes

import pytest

import paper_2407_13996_amd as sg
from test_kv_abi import attend, blocks, commit, kv_map

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def L():
    return sg.lib()


def test_a_views_rows_are_as_wide_as_the_view():
    big = torch.zeros(5, 8, dtype=torch.int32)
    for view, stride in ((big, 8), (big[:, 2:], 8), (big[1:3, 3:7], 8), (big[2:3, 1:6], 5), (big[0:1], 8)):
        b = sg._blocks(view)
        assert (b.table, b.n_requests, b.width) == (view.data_ptr(), view.shape[0], view.shape[1])
        assert b.stride == stride
    for bad in (big.t(), big[:, ::2], big.long(), big.float(), big[0], big[:, :0]):
        with pytest.raises(ValueError):
            sg._blocks(bad)


def test_rows_wider_than_apart_are_refused(L):
    for call in (commit, attend, kv_map):
        for kw in (dict(stride=8, width=8), dict(stride=8, width=3), dict(stride=8, width=0),
                   dict(stride=1 << 31, width=4)):      # rows far apart are no rows of many blocks
            assert call(L, b=blocks(**kw)) == sg.ENODEV, (call, kw)
        for kw in (dict(stride=8, width=9), dict(stride=0, width=1), dict(stride=1 << 27, width=1 << 27)):
            assert call(L, b=blocks(**kw)) == sg.EINVAL, (call, kw)


def test_the_structure_is_the_headers():
    assert ctypes.sizeof(sg.KvBlocks) == 24 and sg.KvBlocks.width.offset == 16
