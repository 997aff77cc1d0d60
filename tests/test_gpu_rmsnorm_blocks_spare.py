"""GPU parity of the norm out as codes with block scales where rows and columns end inside a block: every scale byte is the quantizer's, those of rows that do not exist among them, also
where statistics or weights are not finite."""
import pytest
import torch

from paper_2512_15306_amd import llmq
from tests.test_gpu_rmsnorm_blocks import empty, forward, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,C", [(140, 200), (130, 1001), (257, 4100), (128, 100), (5, 384), (1, 7), (300, 130)])
@pytest.mark.parametrize("what", ["nothing", "a row of NaN", "a row of zeros", "an infinite weight", "a weight of NaN"])
@pytest.mark.parametrize("rows,cols", [(True, True), (False, True), (True, False)])
@pytest.mark.parametrize("fmt", [0, 1])
def test_bytes_of_rows_that_do_not_exist(M, C, what, rows, cols, fmt):
    print("norm spare bytes", M, C, what, rows, cols, fmt, flush=True)
    res, x, w = inputs(M, C, M + C)
    eps = 1e-6
    if what == "a row of NaN":
        res[M - 1, C // 2] = float("nan")
    elif what == "a row of zeros":
        res[M // 2], x[M // 2], eps = 0, 0, 0.0
    elif what != "nothing":
        w[C - 1] = float("inf") if "infinite" in what else float("nan")
    out = forward(res, x, w, fmt, rows, cols, eps=eps)
    q, s, qt, st = empty(M, C, dtype=torch.uint8), empty(llmq.llmq_block_scales_bytes(M, C), dtype=torch.uint8), empty(C, M, dtype=torch.uint8), empty(llmq.llmq_block_scales_bytes(C, M), dtype=torch.uint8)
    llmq.llmq_quantize_fp8_blocks(out["y"], fmt, 1, q, s, qt, st)
    assert torch.isfinite(out["y"]).all() == (what == "nothing")
    if rows:
        assert torch.equal(out["s"], s) and torch.equal(out["q"], q)
    if cols:
        assert torch.equal(out["st"], st) and torch.equal(out["qt"], qt)
