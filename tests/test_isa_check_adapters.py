"""The build's check of copies that are counted by hand, where a loop of matrix instructions with loads of its own stands behind the product: allowed only where no copy can be in flight."""
from paper_2510_25590_amd import isa_check as ic

KERNEL = """
.LBB0_1:
	;;#ASMSTART
	global_load_lds_dwordx4 v1, s[2:3]
	;;#ASMEND
	v_mfma_f32_16x16x32_bf16 v[4:7], v[8:11], v[12:15], v[4:7]
	s_cbranch_scc1 .LBB0_1
	;;#ASMSTART
	s_waitcnt vmcnt(0) lgkmcnt(0)
	;;#ASMEND
.LBB0_2:
	global_load_dwordx4 v[8:11], v[2:3], off
	s_waitcnt vmcnt(0)
	v_mfma_f32_16x16x32_bf16 v[4:7], v[8:11], v[12:15], v[4:7]
	s_cbranch_scc1 .LBB0_2
	s_endpgm
"""


def test_loop_behind_a_wait_for_all_copies_passes():
    assert ic.check_copies("behind", KERNEL.strip().splitlines()) == []


def test_loop_that_copies_may_reach_is_found():
    for was, now in (("vmcnt(0) lgkmcnt(0)", "vmcnt(1) lgkmcnt(0)"), ("vmcnt(0) lgkmcnt(0)", "lgkmcnt(0)"), ("\ts_cbranch_scc1 .LBB0_1\n", "\ts_cbranch_scc1 .LBB0_1\n\ts_cbranch_scc0 .LBB0_2\n")):
        errors = ic.check_copies("reached", KERNEL.replace(was, now, 1).strip().splitlines())
        assert errors and "global_load_dwordx4 v[8:11]" in errors[0], (was, now)


def test_loop_that_holds_a_copy_is_found():
    errors = ic.check_copies("own copy", KERNEL.replace("\tglobal_load_dwordx4 v[8:11]", "\t;;#ASMSTART\n\tglobal_load_lds_dwordx4 v1, s[2:3]\n\t;;#ASMEND\n\tglobal_load_dwordx4 v[8:11]").strip().splitlines())
    assert errors and "global_load_dwordx4 v[8:11]" in errors[0]
