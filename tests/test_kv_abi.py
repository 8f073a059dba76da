"""The cache's calls refuse bad arguments on the host, before any context: no GPU needed."""
import ctypes

import pytest

import paper_2407_13996_amd as sg

NULL = None
r = ctypes.byref


@pytest.fixture(scope="module")
def L():
    return sg.lib()


def cache(**kw):
    a = dict(pool=256, pool_pages=16, layer_stride=0, n_layers=1, page_shift=18, block_tokens=64, kv_heads=8,
             head_dim=128, dtype=sg.BF16)
    a.update(kw)
    return sg.KvCache(**a)


def blocks(**kw):
    a = dict(table=256, stride=8, n_requests=4)
    a.update(kw)
    return sg.KvBlocks(**a)


def rows(**kw):
    a = dict(ptr=256, token_stride=1024, head_stride=128)
    a.update(kw)
    return sg.Rows(**a)


BAD_CACHES = [dict(pool=0), dict(pool=128), dict(pool_pages=0), dict(pool_pages=(1 << 32) + 1), dict(page_shift=9),
              dict(page_shift=31), dict(page_shift=17), dict(block_tokens=8), dict(block_tokens=48),
              dict(block_tokens=2048), dict(kv_heads=0), dict(kv_heads=257), dict(head_dim=80), dict(head_dim=0),
              dict(dtype=sg.F32), dict(dtype=7), dict(n_layers=0),
              dict(n_layers=2, page_shift=19, layer_stride=(1 << 18) - 256),      # layers that overlap
              dict(n_layers=2, page_shift=19, layer_stride=(1 << 18) + 8),        # not a multiple of 256
              dict(n_layers=2, page_shift=19, layer_stride=(1 << 18) + 256),      # the second passes the page
              dict(n_layers=2, layer_stride=(16 << 18) - 256), dict(n_layers=65537, layer_stride=1 << 40)]
BAD_BLOCKS = [dict(table=0), dict(table=258), dict(stride=0), dict(n_requests=0), dict(n_requests=4097),
              dict(stride=1 << 26)]


def append(L, c=None, layer=0, k=None, v=None, slots=256, n=5):
    return L.colored_kv_append(NULL, r(c or cache()), layer, r(k or rows()), r(v or rows()), slots, n, None)


def commit(L, c=None, b=None, lens=256, path=256, stride=4, accepted=256, out=512):
    return L.colored_kv_commit(NULL, r(c or cache()), r(b or blocks()), lens, path, stride, accepted, out, None)


def attend(L, c=None, layer=0, q=None, heads=32, q_start=256, n=5, nodes=4, b=None, lens=256, totals=256, mask=256,
           words=1, scale=0.1, cap=0.0, o=None, lse=256, work=256, bytes_=1 << 40):
    return L.colored_tree_attention(NULL, r(c or cache()), layer, r(q or rows()), heads, q_start, n, nodes,
                                    r(b or blocks()), lens, totals, mask, words, scale, cap, r(o or rows()), lse, work,
                                    bytes_, None)


def kv_map(L, block=16, before=None, after=None, ring=256, size=8, b=None, new=256, q_start=256, slots=256,
           request=256, position=256, n=5):
    before = before or sg.KvState(256, 256, 256)
    after = after or sg.KvState(512, 512, 512)
    return L.colored_kv_map(NULL, block, r(before), r(after), ring, size, r(b or blocks()), new, q_start, slots,
                            request, position, n, None)


def test_sound_arguments_reach_the_context(L):
    assert append(L) == append(L, n=0) == append(L, c=cache(n_layers=2, layer_stride=16 << 18), layer=1) == sg.ENODEV
    assert append(L, c=cache(n_layers=2, page_shift=19, layer_stride=1 << 18), layer=1) == sg.ENODEV
    assert commit(L) == attend(L) == attend(L, n=0) == kv_map(L) == sg.ENODEV
    assert attend(L, mask=None, words=0, lse=None) == sg.ENODEV
    assert kv_map(L, n=0, slots=None, request=None, position=None) == sg.ENODEV


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_bad_caches(L, bad):
    c = cache(**bad)
    assert append(L, c=c) == commit(L, c=c) == attend(L, c=c) == sg.EINVAL
    n = ctypes.c_uint64()
    assert L.sgdrc_tree_attention_workspace(r(c), 32, 4, r(n)) == sg.EINVAL


@pytest.mark.parametrize("bad", BAD_BLOCKS, ids=str)
def test_bad_block_tables(L, bad):
    b = blocks(**bad)
    assert commit(L, b=b) == attend(L, b=b) == sg.EINVAL
    assert kv_map(L, b=blocks(**dict(bad, **({"stride": 1 << 27} if bad.get("stride") else {})))) == sg.EINVAL


@pytest.mark.parametrize("bad", [dict(ptr=0), dict(ptr=264), dict(token_stride=12), dict(head_stride=4),
                                 dict(token_stride=(1 << 30) + 8)], ids=str)
def test_bad_rows(L, bad):
    x = rows(**bad)
    assert append(L, k=x) == append(L, v=x) == attend(L, q=x) == attend(L, o=x) == sg.EINVAL
    assert append(L, k=x, n=0) == attend(L, q=x, n=0) == sg.ENODEV  # nothing to read


def test_other_refusals(L):
    assert append(L, layer=1) == attend(L, layer=1) == sg.EINVAL
    assert append(L, slots=0) == append(L, slots=260) == append(L, n=1 << 31) == sg.EINVAL
    for kw in (dict(lens=0), dict(path=0), dict(accepted=2), dict(out=0), dict(out=256), dict(stride=0),
               dict(stride=257)):
        assert commit(L, **kw) == sg.EINVAL, kw
    for kw in (dict(heads=0), dict(heads=12), dict(heads=1032), dict(nodes=0), dict(nodes=257), dict(words=0),
               dict(words=5), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(q_start=0), dict(lens=0),
               dict(totals=258), dict(mask=260), dict(lse=258), dict(work=0), dict(work=128), dict(bytes_=1024),
               dict(b=blocks(stride=1 << 24, n_requests=4096)), dict(n=1 << 31)):
        assert attend(L, **kw) == sg.EINVAL, kw
    for kw in (dict(block=8), dict(block=24), dict(ring=0), dict(size=0), dict(new=0), dict(q_start=0), dict(slots=0),
               dict(slots=260), dict(request=0), dict(position=0), dict(n=1 << 31),
               dict(before=sg.KvState(0, 256, 256)), dict(after=sg.KvState(516, 512, 512)),
               dict(after=sg.KvState(512, 256, 512)), dict(after=sg.KvState(256, 512, 512))):
        assert kv_map(L, **kw) == sg.EINVAL, kw
    assert L.colored_kv_append(NULL, None, 0, None, None, None, 0, None) == sg.EINVAL
    assert L.sgdrc_tree_attention_workspace(r(cache()), 32, 4, None) == sg.EINVAL


def test_workspace_suffices_and_grows_with_the_rows(L):
    c = cache()
    sizes = [sg.tree_attention_workspace(c, 32, n) for n in (1, 4, 5, 16, 64, 256)]
    assert sizes == sorted(sizes) and sizes[0] >= 2 * 4 * (128 + 2) * 16
    assert attend(L, nodes=4, bytes_=sizes[1]) == sg.ENODEV
    assert attend(L, nodes=4, bytes_=sizes[1] - 1) == sg.EINVAL
