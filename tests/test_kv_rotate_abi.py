"""Rotated cache writes refuse bad arguments on the host, before any context: no GPU needed."""
import ctypes

import pytest

import paper_2407_13996_amd as sg
from test_kv_abi import BAD_CACHES, cache, rows

r = ctypes.byref
torch = pytest.importorskip("torch")


def rotation(**kw):
    a = dict(q_norm=256, k_norm=256, freq=256, norm_dtype=sg.BF16, rot_dims=128, interleaved=0, eps=1e-6)
    a.update(kw)
    return sg.Rotation(**a)


def call(c=None, layer=0, q=None, heads=32, out=None, k=None, v=None, slots=256, position=256, n=5, turn=None):
    return sg.lib().colored_kv_append_rotated(None, r(c or cache()), layer, r(q or rows()), heads, r(out or rows()),
                                              r(k or rows()), r(v or rows()), slots, position, n,
                                              r(turn or rotation()), None)


def test_sound_arguments_reach_the_context():
    assert call() == call(n=0, slots=None) == call(heads=8) == call(heads=1024) == sg.ENODEV
    for kw in (dict(q_norm=None, k_norm=None), dict(freq=None, rot_dims=0), dict(rot_dims=16, interleaved=1),
               dict(norm_dtype=sg.F32, q_norm=260), dict(eps=0.0)):
        assert call(turn=rotation(**kw)) == sg.ENODEV


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_bad_caches(bad):
    assert call(c=cache(**bad)) == sg.EINVAL


@pytest.mark.parametrize("bad", [dict(rot_dims=8), dict(rot_dims=144), dict(rot_dims=100), dict(freq=None),
                                 dict(freq=258), dict(norm_dtype=3), dict(interleaved=2), dict(eps=-1e-6),
                                 dict(eps=float("nan")), dict(eps=float("inf")), dict(q_norm=257),
                                 dict(k_norm=258, norm_dtype=sg.F32)], ids=str)
def test_bad_rotations(bad):
    assert call(turn=rotation(**bad)) == sg.EINVAL


def test_bad_arguments():
    assert sg.lib().colored_kv_append_rotated(None, r(cache()), 0, r(rows()), 8, r(rows()), r(rows()), r(rows()), 256,
                                              256, 1, None, None) == sg.EINVAL
    for kw in (dict(layer=1), dict(heads=0), dict(heads=12), dict(heads=1032), dict(slots=None), dict(slots=260),
               dict(position=None), dict(position=258), dict(n=1 << 31),
               dict(n=(1 << 31) - 1, heads=256, c=cache(kv_heads=256, head_dim=64, block_tokens=16, page_shift=20))):
        assert call(**kw) == sg.EINVAL, kw
    for bad in (dict(ptr=0), dict(ptr=264), dict(token_stride=1020), dict(head_stride=4), dict(token_stride=(1 << 30) + 8)):
        for name in ("q", "out", "k", "v"):
            assert call(**{name: rows(**bad)}) == sg.EINVAL, (name, bad)


def bind(**kw):
    c = sg.kv_cache(256, 1, 12, 16, 1, 64, sg.F16)
    t = torch.zeros(3, 2, 64, dtype=torch.float16)
    a = dict(q=t, k=t[:, :1], v=t[:, 1:], q_out=torch.zeros_like(t), slots=torch.zeros(3, dtype=torch.int64),
             position=torch.zeros(3, dtype=torch.int32), freq=torch.zeros(32), stream=0)
    a.update(kw)
    sg.colored_kv_append_rotated(None, c, 0, **a)


def test_bindings_check_shapes():
    w = torch.zeros(64, dtype=torch.float16)
    t = torch.zeros(3, 2, 64, dtype=torch.float16)
    for kw in (dict(), dict(freq=None), dict(q_norm=w, k_norm=w), dict(k_norm=w.float()), dict(q=t, q_out=t)):
        with pytest.raises(sg.SgdrcError) as e:
            bind(**kw)
        assert e.value.code == sg.ENODEV
    for kw in (dict(q=t[:2]), dict(q_out=torch.zeros(3, 4, 64, dtype=torch.float16)), dict(q=t.float()),
               dict(q_norm=w[:32]), dict(q_norm=w, k_norm=w.float()), dict(q_norm=w.long()), dict(freq=torch.zeros(32).half()),
               dict(freq=torch.zeros(64)[::2]), dict(slots=torch.zeros(3, dtype=torch.int32)),
               dict(position=torch.zeros(3, dtype=torch.int64)), dict(q_out=t[:1].expand(3, 2, 64))):
        with pytest.raises(ValueError):
            bind(**kw)
