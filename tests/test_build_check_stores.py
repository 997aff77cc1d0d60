"""The build's check of wide buffer stores (paper_2512_15306_amd/build.py), on hand-written assembly text: nothing writes a store's registers right behind it."""
import pytest

from paper_2512_15306_amd import build

KERNEL = """_ZN4llmq16gemm_tile_kernelILi0EEEv:                                ; @x
\tv_mov_b32_e32 v40, v41
\tbuffer_store_dwordx4 v[4:7], v1, s[8:11], s4 offen
\tv_add_u32_e32 v8, v7, v9
\tv_mov_b32_e32 v7, v60
\tbuffer_store_dwordx2 v[4:5], v1, s[8:11], s4 offen
\tv_mov_b32_e32 v5, v60
\ts_endpgm
.Lfunc_end0:
"""


@pytest.mark.parametrize("planted", ["\tv_mov_b32_e32 v7, v60", "\tv_lshlrev_b32_e32 v4, 16, v9", "\tv_mov_b64_e32 v[6:7], v[60:61]"])
def test_a_write_right_behind_a_wide_store_fails_the_build(planted):
    build.check_store_data("good.hip", KERNEL)
    anchor = "v[4:7], v1, s[8:11], s4 offen\n"
    with pytest.raises(RuntimeError, match="right behind"):
        build.check_store_data("bad.hip", KERNEL.replace(anchor, anchor + planted + "\n", 1))
