"""CPU check of the 4-bit product's offsets into x: those of lanes without a row of x
stay behind the largest x, whatever columns are added to them, so that the
buffer's own bounds give zeros there.  The source itself, compiled for the host."""
import os
import subprocess

from kernel_asm import CSRC

CHECK = r"""
#include "q4.hip"
// the widest call: 16 rows of 65536 columns; a load begins at one of its 32 columns' first
constexpr uint64_t kBytes = SGDRC_MAX_Q4_BATCH * 65536ull * 2u, kLast = (65536ull - 32u) * 2u;
constexpr bool behind(uint32_t added) { return sgdrc::kQ4Outside + added >= kBytes; }  // (in 32 bits, as the kernel)
constexpr bool all_behind()
{
    for (uint32_t k = 0; k <= kLast; k += 64u)
        if (!behind(k) || !behind(k + 15u))
            return false;
    return true;
}
static_assert(all_behind(), "an offset of a lane without a row lies inside x");
"""


def test_lanes_without_a_row_stay_behind_x(tmp_path):
    from paper_2407_13996_amd import build as B
    src = tmp_path / "offsets.hip"
    src.write_text(CHECK)
    flags = [f for f in B.CFLAGS if f not in ("-fPIC", "-Wall")]
    r = subprocess.run([B.HIPCC, *flags, "-I", CSRC, "-I", os.path.join(os.path.dirname(B.PKG), "include"),
                        "--cuda-host-only", "-fsyntax-only", "-fconstexpr-steps=100000000", str(src)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
