"""The products' loads to LDS set M0 in hand-written assembly, which the compiler cannot be told.  The build checks that it makes
no use of M0 in those kernels; this runs the check, and shows that it notices one."""
import pytest

from paper_2605_06534_amd import build

BY_HAND = "\t;;#ASMSTART\n\ts_mov_b32 m0, s2\n\ts_nop 0\n\tbuffer_load_dwordx4 v4, s[60:63], 0 offen lds\n\t;;#ASMEND\n"


def test_only_the_loads_by_hand_use_m0():
    build.check_m0()


@pytest.mark.parametrize("line", ["s_mov_b32 m0, s3", "s_movreld_b32 s0, s1", "v_movrels_b32_e32 v0, v1", "s_set_gpr_idx_on s0, gpr_idx(SRC0)",
                                  "buffer_load_dword v1, s[0:3], 0 offen lds", "s_sendmsg sendmsg(MSG_INTERRUPT)", "s_add_u32 s0, m0, s1 ; a comment"])
def test_the_check_notices_the_compiler_s_own(line):
    build._check_m0(BY_HAND)
    with pytest.raises(RuntimeError, match="the compiler uses M0"):
        build._check_m0(BY_HAND + "\t" + line + "\n")


def test_the_check_notices_missing_loads():
    with pytest.raises(RuntimeError, match="missing"):
        build._check_m0("\ts_endpgm ; m0\n")
