"""CPU check of the attention kernels that keep values in scratch memory: the
loops over whole steps, where the time goes, have none of it, but for heads of 256,
which read the thread's number back once a step, and for wavefronts with one
block of rows in the form for two, which put one value away a pass."""
import collections
import re

import pytest

import paper_2407_13996_amd as sg
from kernel_asm import device_asm
from test_kv_plan_asm import kernels


def loops(lines):
    """[{opcode: number}] of the instructions in each loop and no inner one of it."""
    out, cur, label = collections.defaultdict(collections.Counter), None, None
    for line in lines:
        m = re.match(r"^(\.LBB\d+_\d+):|^; (%bb\.\d+):", line)
        if m:
            label, cur = m.group(1), None
        m = re.search(r"in Loop: Header=(BB\d+_\d+)", line)
        if m:
            cur = ".L" + m.group(1)
        elif "Loop Header" in line and label:
            cur = label
        m = re.match(r"^\s+([a-z]\w*)", line)
        if m and cur:
            out[cur][m.group(1)] += 1
    return list(out.values())


def number(loop, op):
    return sum(n for name, n in loop.items() if name.startswith(op))


@pytest.mark.parametrize("dtype", [sg.BF16, sg.F16])
@pytest.mark.parametrize("dim,blocks,most", [(128, 2, {1: 2, 2: 0}), (256, 1, {1: 2})])
def test_whole_steps_without_scratch(dtype, dim, blocks, most):
    name = f"k_attend_many<{dtype}, {dim}, {blocks}, 8>"
    lines = next(v for k, v in kernels(device_asm("attention.hip")).items() if name in k)
    step = 2 * (dim // 32) + dim // 16       # products of a block of rows: two K tiles, and V
    # two steps a pass; what masks and counts infinities has more products
    found = {n: x for x in loops(lines) if (n := number(x, "v_mfma") / (2 * step)) in most}
    assert found.keys() == most.keys()
    for n, x in found.items():
        assert number(x, "scratch_") <= most[n], (n, x)
