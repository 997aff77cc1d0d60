"""Host side of the norm with block scales, its gradient and the gated products, without a GPU: sizes and refusals."""
import ctypes

import pytest
import torch

from paper_2512_15306_amd import llmq

P = 0x10000               # never dereferenced: every call below fails validation on the host
BIG = 1 << 20


def test_norm_forward_refuses():
    f = dict(res=P, x=P, w=P, M=4, C=8, eps=1e-6, out=P, rstd=P, fmt=0, q=P, s=P, qt=P, st=P, y=P)

    def call(**o):
        a = dict(f, **o)
        return llmq.lib().llmq_rmsnorm_fwd_fp8_blocks(a["res"], a["x"], a["w"], a["M"], a["C"], a["eps"], a["out"], a["rstd"], a["fmt"], a["q"], a["s"], a["qt"], a["st"], a["y"], None)

    for o in (dict(res=None), dict(w=None), dict(rstd=None), dict(out=None), dict(q=None), dict(s=None), dict(qt=None), dict(st=None), dict(q=None, s=None, qt=None, st=None)):
        assert call(**o) == -1, o
    for o in (dict(M=0), dict(C=0), dict(M=1 << 25), dict(C=1 << 24), dict(M=BIG, C=BIG)):
        assert call(**o) == -2, o
    for eps in (-1e-6, float("nan"), float("inf")):
        assert call(eps=eps) == -8
    assert call(fmt=2) == call(fmt=-1) == -4
    for name in ("res", "x", "w", "out", "rstd", "q", "s", "qt", "st", "y"):
        assert call(**{name: P + 8}) == -3, name
    assert call(x=None, out=P + 8, q=P + 8) == call(x=None, out=None, q=P + 8) == -3          # (without an addition res_out is ignored)


def test_norm_backward_refuses():
    n = llmq.llmq_rmsnorm_bwd_workspace_bytes(4, 8)
    assert n > 0 and llmq.llmq_rmsnorm_bwd_workspace_bytes(0, 8) == llmq.llmq_rmsnorm_bwd_workspace_bytes(4, 1 << 24) == 0
    assert llmq.llmq_rmsnorm_bwd_workspace_bytes(1 << 20, 5120) <= 512 * 5120 * 4 + 4096
    f = dict(dy=P, dres=P, res=P, w=P, rstd=P, M=4, C=8, dx=P, dw=P, fmt=0, amax=P, scale=P, ws=P, bytes=n)

    def call(**o):
        a = dict(f, **o)
        return llmq.lib().llmq_rmsnorm_bwd(a["dy"], a["dres"], a["res"], a["w"], a["rstd"], a["M"], a["C"], a["dx"], a["dw"], 0, a["fmt"], a["amax"], a["scale"], a["ws"], ctypes.c_size_t(a["bytes"]), None)

    for o in (dict(dy=None), dict(res=None), dict(w=None), dict(rstd=None), dict(dx=None), dict(amax=None), dict(ws=None), dict(ws=None, dw=None), dict(ws=None, amax=None, scale=None)):
        assert call(**o) == -1, o
    assert call(M=0) == call(C=-1) == call(C=1 << 24) == call(M=BIG, C=BIG) == -2
    assert call(fmt=2) == -4 and call(bytes=n - 1) == -5
    for name in ("dy", "dres", "res", "w", "dx", "ws"):
        assert call(**{name: P + 8}) == -3, name
    for name in ("rstd", "dw", "amax", "scale"):
        assert call(**{name: P + 2}) == -3, name


@pytest.mark.parametrize("direction", ["fwd", "bwd"])
def test_gated_products_refuse(direction):
    f = dict(A=P, sA=P, fa=0, B=P, sB=P, fb=0, M=4, I=8, T=64, gu=P, out=P, other=P, amax=P)

    def call(**o):
        a = dict(f, **o)
        if direction == "fwd":
            return llmq.lib().llmq_fp8_gemm_blocks_swiglu_fwd(a["A"], a["sA"], a["fa"], a["B"], a["sB"], a["fb"], a["M"], a["I"], a["T"], a["out"], a["gu"], a["amax"], None)
        return llmq.lib().llmq_fp8_gemm_blocks_swiglu_bwd(a["A"], a["sA"], a["fa"], a["B"], a["sB"], a["fb"], a["gu"], a["M"], a["I"], a["T"], a["out"], a["other"], a["amax"], None)

    for name in ("A", "sA", "B", "sB", "out") + (("gu",) if direction == "bwd" else ()):
        assert call(**{name: None}) == -1, name
    for o in (dict(M=0), dict(I=0), dict(T=0), dict(T=15), dict(T=1 << 22), dict(I=1 << 21), dict(M=1 << 31), dict(M=1 << 30, T=1 << 20), dict(M=1 << 30, I=1 << 20), dict(M=1 << 28, I=4096, T=16)):
        assert call(**o) == -2, o
    assert call(fa=2) == call(fb=1) == call(fb=-1) == -4
    for name in ("A", "sA", "B", "sB", "gu", "out") + (("other",) if direction == "bwd" else ()):
        assert call(**{name: P + 8}) == -3, name
    assert call(amax=P + 2) == -3


def test_tensors_on_the_host_are_refused():
    x, u, f = torch.zeros(4, 128, dtype=torch.bfloat16), torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4)
    for call in (lambda: llmq.llmq_fp8_gemm_blocks_swiglu_fwd(u, u, 0, torch.cat((u, u)), u, 0, x[:, :4].contiguous()), lambda: llmq.llmq_fp8_gemm_blocks_swiglu_bwd(u, u, 0, u, u, 0, x[:, :8].contiguous(), x[:, :8].contiguous()),
                 lambda: llmq.llmq_rmsnorm_fwd_fp8_blocks(x, None, x[0], 1e-6, None, f, 0, u, u), lambda: llmq.llmq_rmsnorm_bwd(x, None, x, x[0], f, x, None, False, 0, None, None, None)):
        with pytest.raises(ValueError, match="must live on the GPU"):
            call()
