"""The distance that the build's check of wide buffer stores asks for (paper_2512_15306_amd/build.py), on hand-written assembly text: two wait states, on every path, and both operands of a swap."""
import pytest

from paper_2512_15306_amd import build

STORE = "\tbuffer_store_dwordx4 v[4:7], v1, s[8:11], s4 offen\n"
WRITE = "\tv_mov_b32_e32 v7, v60\n"
OTHER = "\tv_add_u32_e32 v60, v61, v7\n"


def kernel(body):
    return "_ZN4llmq16gemm_tile_kernelILi0EEEv:                                ; @x\n; %bb.0:\n" + body + "\ts_endpgm\n.Lfunc_end0:\n"


@pytest.mark.parametrize("behind", [
    OTHER + WRITE, "\ts_mov_b32 s5, 0\n" + WRITE, "\ts_nop 0\n" + WRITE, "\tv_permlane32_swap_b32_e32 v60, v7\n", "\tv_swap_b32 v61, v4\n", "\tv_permlane16_swap_b32_e32 v6, v60\n", OTHER + "\tv_mov_b64_e32 v[6:7], v[60:61]\n",
    "\ts_cbranch_scc1 .LBB0_2\n" + OTHER + OTHER + "\ts_endpgm\n.LBB0_2:\n" + WRITE,           # where the branch goes to
    "\ts_branch .LBB0_2\n.LBB0_1:\n" + OTHER + "\ts_endpgm\n.LBB0_2:\n" + WRITE,
    ".LBB0_3:                                ; %Flow\n" + OTHER + WRITE])
def test_a_write_within_two_wait_states_fails_the_build(behind):
    with pytest.raises(RuntimeError, match="right behind"):
        build.check_store_data("bad.hip", kernel(STORE + behind), build.STORE_WAIT_STATES)


@pytest.mark.parametrize("behind", [
    OTHER + OTHER + WRITE, "\ts_nop 1\n" + WRITE, "\ts_nop 0\n" + OTHER + WRITE, "\tv_cmp_eq_u32_e32 vcc, v4, v7\n" + OTHER + WRITE, "\tds_read_b128 v[4:7], v9\n", "\tv_readfirstlane_b32 s4, v7\n" + OTHER,
    "\tv_permlane32_swap_b32_e32 v60, v61\n" + OTHER + WRITE,
    "\ts_branch .LBB0_2\n.LBB0_1:\n" + WRITE + "\ts_endpgm\n.LBB0_2:\n" + OTHER,                 # text that is not reached from the store
    OTHER + "\ts_endpgm\n" + WRITE])
def test_what_keeps_its_distance_passes(behind):
    build.check_store_data("good.hip", kernel(STORE + behind), build.STORE_WAIT_STATES)


def test_stores_of_eight_bytes_need_none():
    build.check_store_data("good.hip", kernel("\tbuffer_store_dwordx2 v[6:7], v1, s[8:11], s4 offen\n" + WRITE), build.STORE_WAIT_STATES)
