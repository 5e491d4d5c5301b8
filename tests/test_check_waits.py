"""The check of compiled kernels for registers that are named between a load into them and its wait (no GPU)."""
import os

import pytest

from paper_2007_13055_amd import build, check_waits


def _code(*lines):
    """A function's code as llvm-objdump lists it: (operation, operands[, number of the line that it branches to])."""
    out = ["", "0000000000001000 <kernel>:"]
    for i, line in enumerate(lines):
        target = f" <kernel+0x{8 * line[2]:x}>" if len(line) > 2 and line[2] else " <kernel>" if len(line) > 2 else ""
        out.append(f"\t{line[0]} {line[1]}".ljust(60) + f"// {0x1000 + 8 * i:012X}: DC5C8000 00000002{target}")
    out.append("\ts_endpgm".ljust(60) + f"// {0x1000 + 8 * len(lines):012X}: BF810000")
    return "\n".join(out) + "\n"


def _touched(*lines, every_path=False):
    (name, start, code), = check_waits.kernels(_code(*lines))
    assert name == "kernel" and len(code) == len(lines) + 1
    return [(a - 0x1000) // 8 for a in check_waits.touched_in_flight(start, code, every_path)]


LOAD = ("global_load_dwordx4", "v[2:5], v[0:1], off")
OTHER = ("global_load_dword", "v9, v[0:1], off")


def test_a_copy_in_front_of_the_wait_is_found():
    assert _touched(LOAD, ("v_accvgpr_write_b32", "a63, v5"), ("s_waitcnt", "vmcnt(0)")) == [1]
    assert _touched(LOAD, ("s_waitcnt", "vmcnt(0)"), ("v_accvgpr_write_b32", "a63, v5")) == []
    assert _touched(LOAD, ("s_waitcnt", "lgkmcnt(0)"), ("v_add_f32_e32", "v7, v8, v[4:5]")) == [2]
    assert _touched(LOAD, ("s_waitcnt", "0"), ("v_mov_b32_e32", "v1, v2")) == []
    assert _touched(LOAD, ("v_mov_b32_e32", "v6, v1"), ("v_accvgpr_write_b32", "a5, v1")) == []      # other registers
    assert _touched(("buffer_load_dwordx4", "a[0:3], v1, s[0:3], 0 offen"), ("v_accvgpr_read_b32", "v9, a2")) == [1]


def test_an_address_in_a_register_that_is_still_to_be_filled_is_found():
    assert _touched(LOAD, ("v_lshl_add_u64", "v[2:3], s[0:1], 0, v[6:7]"), ("global_load_dwordx4", "v[10:13], v[2:3], off")) == [1, 2]
    assert _touched(("global_load_dwordx4", "v[0:3], v[0:1], off"), ("s_waitcnt", "vmcnt(0)"), ("v_mov_b32_e32", "v4, v0")) == []   # its own
    assert _touched(LOAD, LOAD, ("s_waitcnt", "vmcnt(0)")) == []         # loads return in order


def test_younger_operations_are_counted():
    store = ("global_store_dword", "v[0:1], v8, off")
    use = ("ds_write_b128", "v20, v[2:5]")
    for younger in (OTHER, store, ("buffer_load_dwordx4", "v30, s[0:3], 0 offen lds")):
        assert _touched(LOAD, younger, ("s_waitcnt", "vmcnt(1)"), use) == []
        assert _touched(LOAD, younger, ("s_waitcnt", "vmcnt(2)"), use) == [3]
    assert _touched(LOAD, OTHER, ("s_waitcnt", "vmcnt(1)"), ("v_mov_b32_e32", "v1, v9")) == [3]


def test_paths():
    use = ("v_mov_b32_e32", "v7, v2")
    # a wait on one of two paths
    skip = (LOAD, ("s_cbranch_scc1", "1", 3), ("s_waitcnt", "vmcnt(0)"), use)
    assert _touched(*skip) == [3] and _touched(*skip, every_path=True) == []
    # around a loop: the load of one trip is waited for in the next, by the count of those behind it
    loop = lambda n: (OTHER, LOAD, ("s_waitcnt", f"vmcnt({n})"), ("v_mov_b32_e32", "v7, v9"), ("s_cbranch_scc0", "65531", 0))  # noqa: E731
    assert _touched(*loop(1)) == [] and _touched(*loop(2)) == [3] and _touched(*loop(2), every_path=True) == [3]
    late = (("v_mov_b32_e32", "v7, v2"), LOAD, ("s_cbranch_scc0", "65531", 0), ("s_waitcnt", "vmcnt(0)"))
    assert _touched(*late) == [0] and _touched(*late, every_path=True) == []                        # not in the first trip


@pytest.mark.parametrize("name", build.NO_SPILL)
def test_built_kernels_wait_for_their_loads(name):
    obj = os.path.join(build.OBJDIR, name + ".o")
    if not os.path.exists(obj):
        pytest.skip("the objects are not kept here; the build itself makes this check")
    assert build._touching_early(name, obj) == {}
