"""The products' loads to LDS set M0 in hand-written assembly, which the compiler cannot be told, and read scalar registers there
that a vector instruction must not have written shortly before.  The build checks both; this runs the checks, and shows that
they notice a violation."""
import pytest

from paper_2605_06534_amd import build

BY_HAND = "\t;;#ASMSTART\n\ts_mov_b32 m0, s2\n\ts_nop 0\n\tbuffer_load_dwordx4 v4, s[60:63], 0 offen lds\n\t;;#ASMEND\n"


def test_what_the_loads_by_hand_assume():
    build.check_loads_to_lds()


@pytest.mark.parametrize("line", ["s_mov_b32 m0, s3", "s_movreld_b32 s0, s1", "v_movrels_b32_e32 v0, v1", "s_set_gpr_idx_on s0, gpr_idx(SRC0)",
                                  "buffer_load_dword v1, s[0:3], 0 offen lds", "s_sendmsg sendmsg(MSG_INTERRUPT)", "s_add_u32 s0, m0, s1 ; a comment"])
def test_the_check_notices_the_compiler_s_own(line):
    build._check_m0(BY_HAND)
    with pytest.raises(RuntimeError, match="the compiler uses M0"):
        build._check_m0(BY_HAND + "\t" + line + "\n")


def test_the_check_notices_missing_loads():
    with pytest.raises(RuntimeError, match="missing"):
        build._check_m0("\ts_endpgm ; m0\n")


@pytest.mark.parametrize("code", ["v_readfirstlane_b32 s60, v1\n{}", "v_readlane_b32 s63, v1, 3\n\ts_nop 1\n{}", "v_cmp_gt_i32_e64 s[62:63], s1, v4\n{}",
                                  "v_add_co_u32_e64 v1, s[60:61], v2, v3\n{}",
                                  ".LBB0_1:\n{}\tv_readfirstlane_b32 s61, v1\n\ts_cbranch_scc1 .LBB0_1\n",
                                  "v_readfirstlane_b32 s61, v1\n\ts_branch .LBB0_2\n.LBB0_1:\n\ts_nop 7\n.LBB0_2:\n{}"])
def test_the_check_notices_scalars_written_shortly_before(code):
    with pytest.raises(RuntimeError, match="too shortly before"):
        build._check_scalar_operands("\t" + code.format(BY_HAND))


@pytest.mark.parametrize("code", ["{}", "v_readfirstlane_b32 s60, v1\n\ts_nop 4\n{}", "v_readfirstlane_b32 s2, v1\n{}", "s_mov_b32 s60, s1\n{}", "v_readfirstlane_b32 s64, v1\n{}",
                                  "v_cmp_gt_i32_e64 s[62:63], s1, v4\n\ts_nop 2\n{}", "v_mov_b32_e32 v4, s60\n{}",
                                  "v_readfirstlane_b32 s61, v1\n\ts_branch .LBB0_2\n.LBB0_1:\n{}.LBB0_2:\n\ts_endpgm\n"])
def test_the_check_lets_others_be(code):
    build._check_scalar_operands("\t" + code.format(BY_HAND))
