"""The calls of 4-bit weights refuse bad arguments on the host, before any context: no GPU needed."""
import ctypes

import numpy as np
import pytest

import paper_2407_13996_amd as sg
import q4_oracle as qo

r = ctypes.byref
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def L():
    return sg.lib()


def q4(**kw):
    a = dict(rows=32, cols=256, group=64, dtype=sg.BF16, zeros=0, reserved=0)
    a.update(kw)
    return sg.Q4(**a)


def paged(**kw):
    a = dict(pool=256, pt=256, pool_pages=4)
    a.update(kw)
    return sg.Paged(**a)


def pack(L, dst=None, q=None, codes=256, stride=256, scales=256, zeros=None, shift=12):
    return L.colored_q4_pack(None, r(dst or paged()), r(q or q4()), codes, stride, scales, zeros, shift, None)


def gemv(L, w=None, q=None, x=256, batch=1, y=256, shift=12):
    return L.colored_gemv_q4(None, r(w or paged()), r(q or q4()), x, batch, y, shift, None)


def test_sound_arguments_reach_the_context(L):
    assert pack(L) == gemv(L) == gemv(L, batch=16) == sg.ENODEV
    assert pack(L, q=q4(zeros=1), zeros=256) == gemv(L, q=q4(zeros=1, cols=65536, dtype=sg.F16)) == sg.ENODEV
    assert pack(L, codes=257, scales=258) == gemv(L, y=260) == sg.ENODEV


@pytest.mark.parametrize("bad", [dict(rows=0), dict(cols=0), dict(cols=96), dict(cols=65600, group=32), dict(group=16),
                                 dict(group=256), dict(group=0), dict(dtype=sg.F32), dict(dtype=7), dict(zeros=2),
                                 dict(reserved=1)], ids=str)
def test_bad_matrices(L, bad):
    n = ctypes.c_uint64()
    q = q4(**bad)
    assert pack(L, q=q, zeros=256 if q.zeros else None, stride=70000) == gemv(L, q=q) == sg.EINVAL
    assert L.sgdrc_q4_bytes(r(q), r(n)) == sg.EINVAL


@pytest.mark.parametrize("bad", [dict(pool=0), dict(pool=128), dict(pt=0), dict(pt=258), dict(pool_pages=0)], ids=str)
def test_bad_pages(L, bad):
    assert pack(L, dst=paged(**bad)) == gemv(L, w=paged(**bad)) == sg.EINVAL


def test_bad_arguments(L):
    for kw in (dict(codes=None), dict(scales=None), dict(scales=257), dict(stride=255), dict(stride=1 << 41),
               dict(zeros=256), dict(q=q4(zeros=1)), dict(q=q4(zeros=1), zeros=257), dict(shift=9), dict(shift=31)):
        assert pack(L, **kw) == sg.EINVAL, kw
    for kw in (dict(x=None), dict(x=264), dict(y=None), dict(y=258), dict(batch=0), dict(batch=17), dict(shift=9)):
        assert gemv(L, **kw) == sg.EINVAL, kw
    assert pack(L, q=q4(rows=1 << 27, cols=1024), stride=1024) == sg.EINVAL     # 2^26 blocks
    assert gemv(L, q=q4(rows=(1 << 32) - 1, cols=1024)) == sg.EINVAL
    n = ctypes.c_uint64()
    assert L.sgdrc_q4_bytes(r(q4()), None) == L.sgdrc_q4_bytes(None, r(n)) == sg.EINVAL
    assert "NULL" in sg.last_error()


def test_bytes():
    for rows, cols, group, zeros in ((1, 32, 32, False), (17, 160, 32, True), (4096, 11008, 128, False)):
        tiles, segs, per = qo.sizes(rows, cols, group)
        assert sg.q4_bytes(sg.q4(rows, cols, group, sg.F16, zeros)) == tiles * segs * (1024 + 32 * per * (1 + zeros))


def test_bindings_check_shapes():
    q = sg.q4(4, 64, 32, sg.F16, True)
    ok = dict(codes=torch.zeros(4, 64, dtype=torch.uint8), scales=torch.zeros(4, 2, dtype=torch.float16),
              zeros=torch.zeros(4, 2, dtype=torch.float16))
    for kw in (dict(codes=torch.zeros(4, 32, dtype=torch.uint8)), dict(codes=torch.zeros(4, 64, dtype=torch.int32)),
               dict(codes=torch.zeros(64, 4, dtype=torch.uint8).t()), dict(scales=torch.zeros(4, 2)),
               dict(scales=torch.zeros(4, 4, dtype=torch.float16)[:, ::2]),
               dict(zeros=torch.zeros(2, 4, dtype=torch.float16)), dict(zeros=torch.zeros(4, 2, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            sg.colored_q4_pack(None, paged(), q, **{**ok, **kw}, page_shift=12, stream=0)
    with pytest.raises(sg.SgdrcError) as e:
        sg.colored_q4_pack(None, paged(), q, **ok, page_shift=12, stream=0)
    assert e.value.code == sg.ENODEV


def test_the_layout_by_hand():
    """One code, one scale: their places as the header gives them."""
    codes = np.zeros((20, 256), dtype=np.uint8)
    codes[17, 128 + 32 * 2 + 8 * 3 + 5] = 11   # block 3, word 2 of piece [3][1], column 5 of eight: bit 24
    s = np.zeros((20, 4), dtype=np.uint16)
    s[17, 3] = 0x1234                          # block 3, [0][1][1]
    out = qo.packed(codes, s, None, 64)
    assert out.nonzero()[0].tolist() == [3 * 1024 + (3 * 16 + 1) * 16 + 2 * 4 + 3, 4 * 1024 + 3 * 64 + 10,
                                         4 * 1024 + 3 * 64 + 11]
    assert out[3 * 1024 + 49 * 16 + 11] == 11


def test_bindings_check_products():
    q = sg.q4(4, 64, 32, sg.F16)
    ok = dict(x=torch.zeros(2, 64, dtype=torch.float16), y=torch.zeros(2, 4))
    for kw in (dict(x=torch.zeros(2, 64, dtype=torch.bfloat16)), dict(x=torch.zeros(1, 64, dtype=torch.float16)),
               dict(x=torch.zeros(2, 128, dtype=torch.float16)[:, ::2]), dict(y=torch.zeros(2, 3)),
               dict(y=torch.zeros(2, 4, dtype=torch.float16)), dict(y=torch.zeros(4, 2).t())):
        with pytest.raises(ValueError):
            sg.colored_gemv_q4(None, paged(), q, batch=2, page_shift=12, stream=0, **{**ok, **kw})
    with pytest.raises(sg.SgdrcError) as e:
        sg.colored_gemv_q4(None, paged(), q, batch=2, page_shift=12, stream=0, **ok)
    assert e.value.code == sg.ENODEV
