"""The build's check of kernels whose output may be one of their inputs (paper_2512_15306_amd/build.py), on hand-written metadata."""
import pytest

from paper_2512_15306_amd import build

METADATA = """\t.amdgpu_metadata
---
amdhsa.kernels:
  - .agpr_count:     8
    .args:
      - .actual_access:  read_only
        .address_space:  global
        .offset:         0
        .size:           8
        .value_kind:     global_buffer
      - .address_space:  global
        .offset:         32
        .size:           8
        .value_kind:     global_buffer
    .name:           _ZN4llmq19gemm_glu_few_kernelE
  - .agpr_count:     256
    .args:
      - .actual_access:  read_only
        .address_space:  global
        .offset:         0
        .size:           8
        .value_kind:     global_buffer
      - .address_space:  global
        .offset:         16
        .size:           8
        .value_kind:     global_buffer
    .name:           _ZN4llmq16gemm_tile_kernelE
...
"""


@pytest.mark.parametrize("offset,kernel", [(32, "gemm_glu_few_kernel"), (16, "gemm_tile_kernel")])
@pytest.mark.parametrize("access", ["write_only", "read_write"])
def test_an_output_declared_apart_fails_the_build(access, offset, kernel):
    build.check_in_place("good.hip", METADATA)
    at = "      - .address_space:  global\n        .offset:         %d" % offset
    bad = METADATA.replace(at, at.replace("- .address_space:", "- .actual_access:  %s\n        .address_space:" % access))
    assert bad != METADATA
    with pytest.raises(RuntimeError, match="%sE: the pointer at %d" % (kernel, offset)):
        build.check_in_place("bad.hip", bad)


def test_without_metadata_nothing_is_known():
    with pytest.raises(RuntimeError, match="no metadata"):
        build.check_in_place("bad.hip", "\ts_endpgm\n")


def test_the_sources_of_the_gradient_are_checked():
    assert build.IN_PLACE_SOURCES == {"gemm_glu_bwd_e4m3_e4m3.hip", "gemm_glu_bwd_e5m2_e4m3.hip"} and build.IN_PLACE_SOURCES <= build.CHECKED_SOURCES
