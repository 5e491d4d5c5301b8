"""What registers the compiled tile kernel takes (no GPU): more of them are fewer wavefronts a SIMD, which wait for memory instead of
working beside one another."""
import os
import re

import pytest

from paper_2007_13055_amd import build, check_waits


def test_plain_tile_kernels_hold_their_sums_and_nothing_else():
    """Without a gate the accumulation registers are those of the sums, 16 a 32x32 tile; fp32 64x64 blocks with two tiles along m
    fill the others, and keep pieces of what is loaded there, too."""
    obj = os.path.join(build.OBJDIR, "bsr_mfma_tile.hip.o")
    if not os.path.exists(obj):
        pytest.skip("the objects are not kept here")
    seen = 0
    for name, taken in check_waits.accumulation_registers(obj).items():
        m = re.search(r"bsr_mfma_tileI(\w+?)Li(\d+)ELi(\d+)ELi(\d)ELi(\d)E\d+(no_epilogue|epilogue_args)", name)
        if not m:
            continue
        bs_r, bs_c, tiles, depth = (int(v) for v in m.groups()[1:5])
        sums = bs_r // 32 * tiles * 16
        assert taken == sums or (m.group(1) == "ff" and (bs_r, bs_c, tiles, depth) == (64, 64, 2, 2)), (name, taken, sums)
        seen += 1
    assert seen > 200
