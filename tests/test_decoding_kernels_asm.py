"""CPU check of the compiled kernels of 4-bit weights, rotated writes and draft
verification: no barrier in a loop that lanes of one wavefront could leave at
different times, and no vector registers in scratch memory but a few in forms of
the 4-bit product with zero points and several row blocks."""
import re

import pytest

from kernel_asm import device_asm, kernel_resources
from test_kernel_cfg import barrier_depths, divergent_barrier_loops

# k_gemv_q4<type, groups of 128 columns, zero points, row blocks, x in LDS>: these hold values of the
# tile loop in scratch, and k_gemv_q4<., 2, true, 2, true> some of a unit's
FEW = re.compile(r"k_gemv_q4<\d, \d, true, [24], (true|false)>")


@pytest.mark.parametrize("src,kernels", [("q4.hip", "k_gemv_q4 k_q4_pack"), ("rotate.hip", "k_kv_rotate"),
                                         ("verify.hip", "k_draft_verify")])
def test_barriers_and_registers(src, kernels):
    asm = device_asm(src)
    assert list(barrier_depths(asm))
    bad = sorted(set(divergent_barrier_loops(asm)))
    assert not bad, f"barrier inside a lane-divergent inner loop in: {bad}"
    found = kernel_resources(asm)
    for k in kernels.split():
        assert any(k in name for name in found)
    for name, r in found.items():
        most = 8 if FEW.search(name) else 0
        assert r.get("vgpr_spill", 0) <= most and r.get("scratch", 0) <= 4 * most, (name, r)
