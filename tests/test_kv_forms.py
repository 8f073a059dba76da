"""The tiles that the cache's calls count on being at work at once: the ranges
that attention cuts its work in, and the writes of up to 2048 tiles of 16 tokens, are at
most as many as the GPU holds workgroups, by the registers and LDS of the
compiled kernels.  No GPU needed."""
import pytest

import paper_2407_13996_amd as sg
from kernel_asm import device_asm, kernel_resources

CUS, LDS, VGPRS = 256, 160 * 1024, 512


def workgroups(r, waves):
    """Of ``waves`` wavefronts, on the whole GPU."""
    regs = -(-r["vgpr"] // 8) * 8
    on_simd = min(VGPRS // regs, 8)
    if r["sgpr"] > 100:
        on_simd = min(on_simd, 7)
    return CUS * min(LDS // r["lds"], on_simd * 4 // waves)


@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("nodes,rows,kernel,waves", [(1, 16, "k_attend_few<{}, {}>", 4), (16, 16, "k_attend_few<{}, {}>", 4),
                                                     (17, 64, "k_attend_many<{}, {}, 1, 4>", 4),
                                                     (64, 64, "k_attend_many<{}, {}, 1, 4>", 4),
                                                     (128, 128, "k_attend_many<{}, {}, 1, 8>", 8),
                                                     (256, 256, "k_attend_many<{}, {}, 2, 8>", 8)])
def test_all_ranges_are_at_work_at_once(dim, nodes, rows, kernel, waves):
    if dim == 256 and rows == 256:
        rows, kernel = 128, "k_attend_many<{}, {}, 1, 8>"
    cache = sg.KvCache(pool=256, pool_pages=16, layer_stride=0, n_layers=1, page_shift=18, block_tokens=64, kv_heads=1,
                       head_dim=dim, dtype=sg.BF16)
    ranges, rest = divmod(sg.tree_attention_workspace(cache, 1, nodes), 2 * rows * (dim + 2) * 4)
    assert rest == 0
    found = kernel_resources(device_asm("attention.hip"))
    for dtype in (sg.BF16, sg.F16):
        r = next(r for name, r in found.items() if kernel.format(dtype, dim) in name)
        assert 0 < ranges <= workgroups(r, waves), (ranges, r)


def test_tiles_of_16_tokens_are_written_at_once():
    found = {n: r for n, r in kernel_resources(device_asm("kv_cache.hip")).items() if "k_kv_append<" in n and ", 16>" in n}
    assert len(found) == 4
    for name, r in found.items():
        assert workgroups(r, 4) >= 2048, (name, r)
