"""The build's guard of loads that are waited for by their number (weights that stream past few rows), without a GPU."""
import pytest

from paper_2505_11076_amd import build as Bd

BEGIN, END = Bd.PART_MARKS


def kernel(args, part, wait, before=3, inside=4):
    def once(waits):
        return "\t%s\n%s\t%s\n%s" % (BEGIN, "".join("\t%s\n" % l for l in part), END, "\ts_waitcnt %s\n" % wait if waits else "")

    return "_ZN12_GLOBAL__N_123dbf_dense_stream_kernelI%sEEvNS_9DenseArgsE:\n%s.LBB0_1:\n%s\ts_cbranch_scc0 .LBB0_1\n\ts_endpgm\n" % (args, once(False) * before, once(True) * inside)


BYTE, LDS, NUMBER = "global_load_ubyte v1, v[2:3], off", "global_load_lds_dwordx4 v[4:5], off nt", "global_load_dword v1, v[2:3], off"
PLAIN = [BYTE] + [LDS] * 4              # one matrix, two steps, scales of a byte
GATED = [NUMBER, LDS, NUMBER] + [LDS] * 3   # two matrices, a step, scales of 32 bits


def test_kernels_that_load_what_they_wait_for():
    code = kernel("Li3ELb0ELb0ELb0ELi8ELi2E", PLAIN, "vmcnt(15) lgkmcnt(0)") + kernel("Li3ELb1ELb1ELb1ELi8ELi1E", GATED, "vmcnt(18) lgkmcnt(0)", inside=8)
    code += kernel("Li0ELb0ELb0ELb0ELi2ELi2E", [LDS] * 4, "vmcnt(12) lgkmcnt(0)") + kernel("Li3ELb0ELb0ELb0ELi8ELi2E", PLAIN + [LDS], "vmcnt(0)")   # (more loads, longer waits)
    assert Bd._part_loads_report(code, 3) == (4, [])
    assert Bd._part_loads_report("nothing here", 3) == (0, [])


@pytest.mark.parametrize("part,wait,inside,what", [
    (PLAIN[1:], "vmcnt(15)", 4, "4 loads in part 1, of 5"), (["s_load_dword s4, s[2:3], 0x0"] + PLAIN[1:], "vmcnt(15)", 4, "4 loads in part 7, of 5"),
    ([PLAIN[0], "s_cbranch_vccz .LBB0_2"] + PLAIN[1:], "vmcnt(15)", 4, "straight code"), (PLAIN[:2] + [".LBB0_2:  ; in the loop"] + PLAIN[2:], "vmcnt(15)", 4, "straight code"), (PLAIN, "vmcnt(16)", 4, "no wait for all but 15 loads behind part 4"),
    (PLAIN, "lgkmcnt(0)", 4, "no wait for all but 15 loads behind part 7"), (PLAIN, "vmcnt(15)", 3, "6 parts, of 3 before the loop and 4 in it")])
def test_the_build_refuses_fewer(part, wait, inside, what):
    seen, bad = Bd._part_loads_report(kernel("Li3ELb0ELb0ELb0ELi8ELi2E", part, wait, inside=inside), 3)
    assert seen == 1 and any(what in b for b in bad), bad


def test_the_kernels_as_they_are_built():
    Bd._check_part_loads()
