"""CPU check of the compiled kernels that first go through all requests of a
call: a workgroup that has no tile, as every one outside a stream's CU mask, can leave
without that (its CU and L2 are another stream's)."""
import re

import pytest

from kernel_asm import demangle, device_asm


def kernels(asm):
    """{kernel: its lines}"""
    out, cur = {}, None
    for line in asm.splitlines():
        m = re.match(r"^(_Z\w+):", line)
        if m:
            cur = out.setdefault(m.group(1), [])
        elif line.startswith(".Lfunc_end"):
            cur = None
        elif cur is not None:
            cur.append(line)
    return dict(zip(demangle(list(out)), out.values()))


def leaves_without(lines, op):
    """Whether some way from the first instruction to the end meets no ``op``."""
    labels = {m.group(1): i for i, l in enumerate(lines) if (m := re.match(r"^(\.LBB\d+_\d+):", l))}
    todo, seen = [0], set()
    while todo:
        i = todo.pop()
        while i < len(lines) and i not in seen:
            seen.add(i)
            m = re.match(r"^\s+([a-z]\w*)\s*(\S*)", lines[i])
            name, to = m.groups() if m else ("", "")
            if name == "s_endpgm":
                return True
            assert name != "s_setpc_b64", "an indirect jump"
            if name.startswith(op):
                break
            if name.startswith("s_cbranch"):
                todo.append(labels[to])
            elif name == "s_branch":
                todo.append(labels[to])
                break
            i += 1
    return False


def test_the_check_on_hand_made_code():
    def code(branch):
        return ["\ts_mov_b32 s0, 0", f"\t{branch} .LBB0_2" if branch else "\ts_nop 0", ".LBB0_1:",
                "\tds_bpermute_b32 v0, v1, v2", ".LBB0_2:", "\ts_endpgm"]
    assert not leaves_without(code(""), "ds_bpermute")
    assert leaves_without(code("s_cbranch_scc1"), "ds_bpermute") and leaves_without(code("s_branch"), "ds_bpermute")
    assert leaves_without(code(""), "v_mfma")


@pytest.mark.parametrize("src,what", [("kv_cache.hip", "k_kv_map"), ("attention.hip", "k_attend_")])
def test_no_plan_without_a_tile(src, what):
    """(The plan's running sums over a wavefront are exchanges between lanes.)"""
    found = {k: v for k, v in kernels(device_asm(src)).items() if what in k}
    assert found
    for name, lines in found.items():
        assert any("ds_bpermute" in line for line in lines), name
        assert leaves_without(lines, "ds_bpermute"), name
