"""The build's check of the tile kernels' counted waits (paper_2512_15306_amd/build.py), on hand-written assembly text: the N newest requests hold no load to LDS that has to have landed."""
import pytest

from paper_2512_15306_amd import build

TWO = "_ZN4llmq16gemm_tile_kernelILi0ELi0ELi2ELi2ELb1ENS_9GluTuningILi1ENS_10GemmTuningELi1ELb0EEELb0ELb0ELi0ELi1EEEvPKhS5_"
FOUR = TWO.replace("10GemmTuning", "14GemmDeepTuning")
LDS = "\tbuffer_load_dwordx4 v2, s[8:11], s4 offen lds\n"
SCALE = "\tbuffer_load_dword v9, v3, s[12:15], s5 offen\n"


def wait(n):
    return "\t;;#ASMSTART\n\ts_waitcnt vmcnt(%d)\n\t;;#ASMEND\n\ts_barrier\n" % n


def kernel(name, stages, scales, counted, first=None, head="", loop=None, tail=""):
    """A prologue of `stages` slabs of three loads and then `scales` others, a loop of a counted wait, a slab and the others, and `tail`; the waits count `counted` others."""
    in_flight = 3 * (stages - 2)
    step = wait(in_flight + counted) + LDS * 3 + SCALE * scales
    return ("%s:                                ; @x\n; %%bb.0:\n" % name + head + SCALE * scales + LDS * 3 * stages + SCALE * scales + wait(3 * (stages - 1) + (counted if first is None else first))
            + ".LBB0_1:                                ; =>This Inner Loop Header: Depth=1\n" + (step if loop is None else loop) + "\ts_cbranch_scc1 .LBB0_1\n" + tail + wait(0) + "\ts_endpgm\n.Lfunc_end0:\n")


@pytest.mark.parametrize("name,stages", [(TWO, 2), (FOUR, 4)])
@pytest.mark.parametrize("scales", [0, 2, 5])
def test_waits_that_count_what_is_there_pass(name, stages, scales):
    assert build.check_counted_waits("good.hip", kernel(name, stages, scales, scales)) == 1
    assert build.check_counted_waits("good.hip", kernel(name, stages, scales + 1, scales)) == 1           # more loads than counted: a longer wait


@pytest.mark.parametrize("name,stages", [(TWO, 2), (FOUR, 4)])
def test_a_load_less_than_counted_fails_the_build(name, stages):
    with pytest.raises(RuntimeError, match="counted wait"):
        build.check_counted_waits("bad.hip", kernel(name, stages, 4, 5))
    with pytest.raises(RuntimeError, match=r"vmcnt\(%d\)" % (3 * (stages - 1) + 3)):
        build.check_counted_waits("bad.hip", kernel(name, stages, 2, 2, first=3))


def test_a_load_to_lds_behind_the_others_fails_the_build():
    """The order counts, in the loop too."""
    with pytest.raises(RuntimeError, match="counted wait"):
        build.check_counted_waits("bad.hip", kernel(TWO, 2, 2, 2, loop=wait(2) + LDS * 2 + SCALE * 2 + LDS))
    good = kernel(TWO, 2, 2, 2)
    with pytest.raises(RuntimeError, match="counted wait"):
        build.check_counted_waits("bad.hip", good.replace(LDS * 3 + SCALE * 2 + wait(5), LDS * 2 + SCALE + LDS + SCALE + wait(5), 1))


def test_a_path_with_a_load_less_fails_the_build():
    skipped = wait(2) + LDS * 3 + SCALE + "\ts_cbranch_vccz .LBB0_2\n" + SCALE + ".LBB0_2:\n"
    with pytest.raises(RuntimeError, match="counted wait"):
        build.check_counted_waits("bad.hip", kernel(TWO, 2, 2, 2, loop=skipped))
    dead = kernel(TWO, 2, 2, 2, tail=wait(2) + LDS * 3 + wait(2))                                           # behind the loop nobody needs the others
    with pytest.raises(RuntimeError, match="counted wait"):
        build.check_counted_waits("bad.hip", dead)


def test_kernels_without_loads_to_lds_are_none_of_its_business():
    assert build.check_counted_waits("good.hip", kernel(TWO, 2, 2, 2).replace(LDS, SCALE)) == 0


MINI = "_ZN4llmq16gemm_mini_kernelILi0ELi0ELi32ELb1EEEvPKhS2_PtiiiPKfS5_iPjiiiiii"


def mini(tail):
    """Four stages of two slab loads and three others, which the loop's and the last stages' waits count together."""
    stage = SCALE * 3 + LDS * 2
    return ("%s:                                ; @x\n; %%bb.0:\n" % MINI + stage * 4 + "\ts_cbranch_scc1 .LBB0_2\n.LBB0_1:\n" + (wait(15) + stage) * 4 + "\ts_cbranch_scc1 .LBB0_1\n.LBB0_2:\n" + tail + wait(0)
            + "\ts_endpgm\n.Lfunc_end0:\n")


def test_last_stages_whose_codes_nobody_needs():
    assert build.check_counted_waits("good.hip", mini(wait(15) + wait(10) + wait(5))) == 1
    with pytest.raises(RuntimeError, match="counted wait"):
        build.check_counted_waits("bad.hip", mini(wait(15) + LDS * 2 + wait(15)))


BLOCKS, GLU = "_ZN4llmq22gemm_blocks_few_kernelILi0ELi0ELi1ELi2ELb1EEEvPKhS2_S2_S2_PtiiiiPj", "_ZN4llmq19gemm_glu_few_kernelILi0ELi0ELi1ELi1ELi2ELi1ELi3ELb1EEEvPKhS2_S2_S2_PtNS_7GluPlanEiiiPj"


def few(name, *counts):
    return "%s:                                ; @x\n; %%bb.0:\n" % name + "".join(SCALE * 3 + LDS * 6 + wait(n) for n in counts) + wait(0) + "\ts_endpgm\n.Lfunc_end0:\n"


@pytest.mark.parametrize("name,good,bad", [(BLOCKS, (27, 27, 27, 27, 27, 18, 9), (27, 27, 27, 27, 27, 27, 27)), (BLOCKS, (27, 18, 9), (27, 18)), (GLU, (18, 18, 18, 18, 9), (18, 18, 18, 18, 18)), (GLU, (9, 18), (9, 18, 15))])
def test_last_steps_of_the_kernels_for_few_rows(name, good, bad):
    assert build.check_few_rows_waits("good.hip", few(name, *good)) == 1
    with pytest.raises(RuntimeError, match="steps in flight"):
        build.check_few_rows_waits("bad.hip", few(name, *bad))
    assert build.check_few_rows_waits("good.hip", few(name, *bad).replace(LDS, SCALE)) == 0
