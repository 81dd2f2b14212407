"""The build's scan for spilled registers, on every kernel that gathers rows into LDS."""
import pytest

from paper_2509_16518_amd import build

GATHER = "\tglobal_load_lds_dwordx4 v7, s[4:5]\n"


def listing(kernels):
    """Assembly with a function and its metadata for each (name, has a gather, spilled registers)."""
    text = "".join("%s:                 ; @%s\n%s\ts_endpgm\n.Lfunc_end%d:\n" % (k, k, GATHER if g else "", n) for n, (k, g, _) in enumerate(kernels))
    return text + "".join("    .name:           %s\n    .vgpr_count:     256\n    .vgpr_spill_count: %d\n" % (k, s) for k, _, s in kernels)


DQ, RINGS, RESIDENT = "_ZN3fgx9dq_kernelILi128ELb1EEEvNS_7BwdArgsE", "_ZN3fgx12cross_kernelILi128ELi8ELb1ELb0EEEvNS_9CrossArgsE", \
    "_ZN3fgx12cross_kernelILi128ELi8ELb0ELb0EEEvNS_9CrossArgsE"
SMALL, SUMS = "_ZN3fgx12cross_kernelILi64ELi8ELb1ELb0EEEvNS_9CrossArgsE", "_ZN3fgx10sum_kernelILi128EEEvNS_7BwdArgsE"


@pytest.mark.parametrize("kernels", [[(DQ, True, 0)], [(RINGS, True, 1), (RESIDENT, True, 6), (SMALL, True, 0)], [(SUMS, False, 9), (DQ, True, 0)]])
def test_spills_that_are_known(tmp_path, kernels):
    path = tmp_path / "piece.s"
    path.write_text(listing(kernels))
    build.check_spills(str(path))


@pytest.mark.parametrize("kernels", [[(DQ, True, 1)], [(RINGS, True, 2)], [(RESIDENT, True, 7)], [(SMALL, True, 1)], [(SUMS, False, 9), (SUMS + "b", True, 9)],
                                     [(DQ, True, 0), ("_ZN2fg17fgattn_fwd_kernelILi64E", False, 2)]])
def test_spills_that_are_not(tmp_path, kernels):
    path = tmp_path / "piece.s"
    path.write_text(listing(kernels))
    with pytest.raises(RuntimeError):
        build.check_spills(str(path))
