"""The build step's look at the emitted code of the products (host logic only: the assembly is made up here)."""
import pytest

from paper_2201_12023_amd import build as B

NAME = "_ZN4alpa14product_kernelIfLi0ELi0ELi256ELi256ELi2ELi4ELi0ELi0EEEvNS_11ProductArgsE"
LOAD = ["\t;;#ASMSTART", "\ts_mov_b32 m0, s69", "\ts_nop 0", "\tbuffer_load_dwordx4 v4, s[28:31], 0 offen lds", "\t;;#ASMEND"]


def bad(*lines, name=NAME):
    text = "\n".join(["\t.text", f"{name}: ; @{name}", "; %bb.0:", *lines, *LOAD, "\ts_endpgm", ".Lfunc_end0:", "\t.size x", ""])
    return len(B.check_load_ranges(text))


@pytest.mark.parametrize("write", ["v_readfirstlane_b32 s28, v3", "v_readlane_b32 s31, v3, 4", "v_cmp_gt_i32_e64 s[30:31], s69, v2",
                                   "v_mad_u64_u32 v[2:3], s[28:29], v3, s14, v[2:3]", "v_add_co_u32_e64 v1, s[30:31], v2, v3"])
def test_vector_writes_of_a_load_s_range_keep_five_states_away(write):
    far = ["\ts_add_u32 s1, s2, s3"] * 3                # three and the two in front of the load itself
    assert bad("\t" + write) == 1
    assert bad("\t" + write, *far[:2]) == 1
    assert bad("\t" + write, *far) == 0
    assert bad("\t" + write, "\ts_nop 2") == 0 and bad("\t" + write, "\ts_nop 1") == 1
    assert bad("\t" + write, "; a comment", ".LBB0_1:                                ; =>This Inner Loop Header", "; %bb.2:") == 1


def test_other_instructions_may_stand_there():
    assert bad("\tv_readfirstlane_b32 s69, v3") == 0            # the place in LDS, which a scalar instruction reads
    assert bad("\ts_add_u32 s28, s28, s4") == 0
    assert bad("\tv_add_u32_e32 v4, s28, v3") == 0 and bad("\tv_cndmask_b32_e64 v4, v1, v2, s[28:29]") == 0
    assert bad("\tv_readfirstlane_b32 s28, v3", name="_ZN4alpa11pack_kernelIfEEvNS_8PackArgsE") == 0


def test_writes_in_front_of_a_jump_count():
    write = "\tv_readfirstlane_b32 s28, v3"
    loop = [write, "\ts_cbranch_scc1 .LBB0_7", "\ts_endpgm", ".LBB0_7:"]
    assert bad(*loop) == 1
    assert bad(write, "\ts_nop 1", *loop[1:]) == 0
    # a path that is not one: the line above the label does not fall through
    assert bad("\ts_branch .LBB0_9", write, "\ts_endpgm", ".LBB0_7:") == 0
    # a jump back from behind the load
    text = "\n".join([f"{NAME}:", "\ts_nop 7", ".LBB0_1:", *LOAD, write, "\ts_cbranch_scc1 .LBB0_1", "\ts_endpgm", ".Lfunc_end0:", ""])
    assert len(B.check_load_ranges("\n" + text)) == 1
