"""The build's check of the offsets of buffer stores (paper_2512_15306_amd/build.py), on hand-written assembly text: what tells rows behind an output is the lane's offset."""
import pytest

from paper_2512_15306_amd import build

KERNEL = """_ZN4llmq16gemm_tile_kernelILi0EEEv:                                ; @x
\tbuffer_load_dwordx4 v[4:7], v1, s[8:11], s4 offen
\tbuffer_store_dwordx4 v[4:7], v1, s[8:11], 0 offen
\tbuffer_store_short v4, v1, s[8:11], 0 offen offset:32 ; 2 bytes
\tbuffer_store_short_d16_hi v4, v1, s[8:11], 0 offen nt
\tglobal_store_dwordx4 v[40:41], v[4:7], s[8:9]
\ts_endpgm
.Lfunc_end0:
"""


@pytest.mark.parametrize("planted", ["\tbuffer_store_short v4, v1, s[8:11], s4 offen", "\tbuffer_store_dwordx4 v[4:7], v1, s[8:11], s33 offen offset:16", "\tbuffer_store_short_d16_hi v4, v1, s[8:11], s4 offen nt",
                                     "\tbuffer_store_dword v4, off, s[8:11], s4", "\tbuffer_store_byte a4, v1, s[96:99], m0 offen"])
def test_a_store_with_a_scalar_offset_fails_the_build(planted):
    build.check_store_offsets("good.hip", KERNEL)
    with pytest.raises(RuntimeError, match="scalar offset"):
        build.check_store_offsets("bad.hip", KERNEL.replace("\ts_endpgm", planted + "\n\ts_endpgm", 1))
