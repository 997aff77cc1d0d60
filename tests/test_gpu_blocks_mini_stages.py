"""The small-tile kernels of the block-scaled contraction around the number of K steps that they keep on their way: the bytes of the tile kernel."""
import numpy as np
import pytest
import torch

from paper_2512_15306_amd import llmq
from tests import blocks_common as bc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def operand(g, rows, T):
    b = torch.randint(120, 130, (rows, bc.padded(T) // 128), generator=g).numpy()
    return torch.randn(rows, T, generator=g).mul(30).to(bc.FLOAT8[0]).view(torch.uint8).to(DEV), bc.packed(np.asarray(b)).to(DEV)


@pytest.mark.parametrize("T", [128 * k for k in range(1, 18)] + [528, 656, 1040, 1552, 2064, 4000, 4608])
@pytest.mark.parametrize("R,C", [(256, 192), (133, 72)])
def test_the_bytes_of_the_tile_kernel(monkeypatch, R, C, T):
    print("blocks mini", R, C, T, flush=True)
    g = torch.Generator().manual_seed(R + T)
    (a, sa), (b, sb) = operand(g, R, T), operand(g, C, T)
    got = []
    for side in ("0", "32", "64"):
        monkeypatch.setenv("LLMQ_GEMM_MINI", side)
        c, amax = torch.zeros(R, C, device=DEV, dtype=torch.bfloat16), torch.zeros(1, device=DEV)
        for _ in range(3):
            llmq.llmq_fp8_gemm_blocks(a, sa, 0, b, sb, 0, c, False, amax)
        llmq.llmq_fp8_gemm_blocks(a, sa, 0, b, sb, 0, c, True, amax)
        got.append((c, amax))
    assert all(torch.equal(c, got[0][0]) and torch.equal(m, got[0][1]) for c, m in got[1:])
