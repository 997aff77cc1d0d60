"""Query and key norms at the ends of what the call takes: heads whose mean square is a subnormal number, eps, buffers that must not be the same."""
import numpy as np
import pytest
import torch

from paper_2512_15306_amd import llmq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
f64 = lambda t: t.detach().cpu().to(torch.float64).numpy()  # noqa: E731


@pytest.mark.parametrize("D", [128, 64, 100])
def test_small_heads_without_eps(D):
    """Values of about 2^-60 to 2^-70, squares from 0.74 2^-140 on: the mean of a head's squares is a normal number for the first rows and a subnormal one, in steps of 2^-149, for the others.  There each of the D
    multiply-adds is off by half a step at most (sums of such numbers are exact), D 2^-150 of a sum of 0.74 D 2^-140 or more, and the mean by another 2^-150 of 0.74 2^-140: 2.8 2^-10 together, which the
    root halves: less than 2^-9."""
    M = 11
    g = torch.Generator().manual_seed(D)
    rows = torch.exp2(-60.0 - torch.arange(M).double())[:, None]
    x = ((0.75 + torch.rand(M, 3 * D, generator=g).double() / 2).sqrt() * torch.sign(torch.randn(M, 3 * D, generator=g)) * rows).to(torch.bfloat16)
    x = torch.where(x == 0, rows.to(torch.bfloat16), x).to(DEV)
    w = torch.ones(D, device=DEV, dtype=torch.bfloat16)
    q, k = (torch.full((M, D), 7.0, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    rstd = torch.zeros(M, 2, device=DEV)
    llmq.llmq_qk_norm_rope_fwd(x, 1, 1, D, w, w, 0.0, None, None, False, q, k, rstd)
    heads = f64(x)[:, : 2 * D].reshape(M, 2, D)
    r = 1.0 / np.sqrt((heads * heads).mean(-1))
    y = heads * r[..., None]                              # (no pairs are turned)
    got = np.stack([f64(q), f64(k)], 1)
    assert (np.abs(f64(rstd) - r) <= 2.0 ** -9 * r).all(), np.abs(f64(rstd) / r - 1).max()
    assert (np.abs(got - y) <= (2.0 ** -8 + 2.0 ** -9) * (1 + 2.0 ** -8) * np.abs(y)).all()
