"""CPU check of the cache's compiled kernels: no barrier in a loop that lanes
of one wavefront could leave at different times, and no spilled vector
registers but in the attention forms that hold the most rows."""

import pytest

from kernel_asm import device_asm, kernel_resources
from test_kernel_cfg import barrier_depths, divergent_barrier_loops

# the forms of 256 rows (a state of 32 rows a wavefront) and of heads 256 wide
# keep what the rare steps need in scratch memory
SPILLS = ("k_attend_many<1, 128, 2, 8>", "k_attend_many<2, 128, 2, 8>", "k_attend_many<1, 256, 1, 8>",
          "k_attend_many<2, 256, 1, 8>")


@pytest.mark.parametrize("src", ["kv_cache.hip", "attention.hip"])
def test_barriers_and_registers(src):
    asm = device_asm(src)
    assert list(barrier_depths(asm))
    bad = sorted(set(divergent_barrier_loops(asm)))
    assert not bad, f"barrier inside a lane-divergent inner loop in: {bad}"
    kernels = kernel_resources(asm)
    assert kernels
    for name, r in kernels.items():
        if not any(s in name for s in SPILLS):
            assert r.get("vgpr_spill", 0) == 0 and r.get("scratch", 0) == 0, (name, r)
