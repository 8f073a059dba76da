"""CPU check of the 4-bit product's forms that keep values in scratch memory: which they are, how many values,
and that the loop with the products reads none but in the form with two row blocks for groups of 64 with zero points."""
import re

import pytest

import paper_2407_13996_amd as sg
from kernel_asm import device_asm, kernel_resources
from test_kv_plan_asm import kernels
from test_kv_spills_asm import loops, number

# k_gemv_q4<type, groups of 128 columns, zero points, row blocks, x in LDS>: vector registers put away at most
MOST = {(1, 4): 6, (2, 4): 3, (4, 4): 1, (2, 2): 6}
FORM = r"k_gemv_q4<{}, (\d), (true|false), (\d), (?:true|false)>"


@pytest.mark.parametrize("dtype", [sg.BF16, sg.F16])
def test_few_values_and_none_in_the_loop(dtype):
    asm = device_asm("q4.hip")
    seen = 0
    for name, r in kernel_resources(asm).items():
        m = re.search(FORM.format(dtype), name)
        if m:
            per, zeros, blocks = int(m[1]), m[2] == "true", int(m[3])
            most = MOST.get((per, blocks), 0) if zeros else 0
            assert r["vgpr_spill"] <= most, (name, r)
            seen += 1
    assert seen == 24
    for name, lines in kernels(asm).items():
        m = re.search(FORM.format(dtype), name)
        if m:
            most = 12 if (m[1], m[2], m[3]) == ("2", "true", "2") else 0
            inner = [x for x in loops(lines) if number(x, "v_mfma")]
            assert inner, name
            for x in inner:
                assert number(x, "scratch_load") <= most and number(x, "scratch_store") == 0, (name, x)
