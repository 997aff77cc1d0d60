"""Contractions with block scales at the ends of what their generic kernel takes."""
import pytest
import torch

from paper_2512_15306_amd import llmq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("R,C", [((1 << 21) - 1, 1), (3, (1 << 23) + 5)])
def test_the_longest_grid(R, C):
    """8 contraction bytes: 65536 workgroups along the second dimension of the grid, the most it has, and many along the first.  Products of whole numbers up to 7, so every sum is a whole number up to 392, times
    a power of two: exact in binary32 and off by half a step of BF16 at most."""
    g = torch.Generator(DEV).manual_seed(1)
    a, b = (torch.randint(-7, 8, (n, 8), device=DEV, generator=g).float() for n in (R, C))
    sa, sb = (torch.full((llmq.llmq_block_scales_bytes(n, 8),), code, device=DEV, dtype=torch.uint8) for n, code in ((R, 129), (C, 126)))
    c = torch.full((R, C), -3.0, device=DEV, dtype=torch.bfloat16)
    amax = torch.zeros(1, device=DEV)
    llmq.llmq_fp8_gemm_blocks(a.to(torch.float8_e4m3fn).view(torch.uint8), sa, llmq.E4M3, b.to(torch.float8_e4m3fn).view(torch.uint8), sb, llmq.E4M3, c, False, amax)
    want = sum(a[:, k, None] * b[None, :, k] for k in range(8)) * 2.0                # 2^(129 - 127) 2^(126 - 127)
    assert torch.equal(c, want.to(torch.bfloat16)) and amax.item() == c.abs().max().item()
