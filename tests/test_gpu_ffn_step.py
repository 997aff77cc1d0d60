"""The second half of a transformer block as a training step uses it: residual RMSNorm out as codes with block scales, gate and up products joined with the SwiGLU, the down product; backwards the gradient of the
joined products, block-scaled input and weight gradients added up over two micro-steps, and the gradient of the residual RMSNorm.  Every stage is checked on what the stage before it left; the same
step on another stream, from a graph, beside another one, and as the separate operators that it joins."""
import numpy as np
import pytest
import torch

from paper_2512_15306_amd import llmq
from tests import blocks_common as bc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6
f64 = lambda t: t.detach().cpu().to(torch.float64).numpy()  # noqa: E731
bf = lambda *n: torch.zeros(*n, device=DEV, dtype=torch.bfloat16)  # noqa: E731
u8 = lambda *n: torch.zeros(*n, device=DEV, dtype=torch.uint8)  # noqa: E731
f32 = lambda *n: torch.zeros(*n, device=DEV)  # noqa: E731


class Codes:
    """Both copies of a tensor in blocks."""

    def __init__(self, rows, cols, fmt, block_rows):
        self.fmt, self.block_rows = fmt, block_rows
        self.q, self.q_t = u8(rows, cols), u8(cols, rows)
        self.s, self.s_t = u8(llmq.llmq_block_scales_bytes(rows, cols)), u8(llmq.llmq_block_scales_bytes(cols, rows))

    def of(self, x):
        llmq.llmq_quantize_fp8_blocks(x, self.fmt, self.block_rows, self.q, self.s, self.q_t, self.s_t)
        return self

    def values(self, transposed=False):
        q, s = (self.q_t, self.s_t) if transposed else (self.q, self.s)
        return bc.values(bc.decode(q, self.fmt), bc.scale_bytes(s, *q.shape))


class Half:
    """M tokens of C columns, I columns between the products"""

    def __init__(self, M, C, I, seed):
        g = torch.Generator().manual_seed(seed)
        rand = lambda *n, std=1.0: torch.randn(*n, generator=g).mul(std).to(torch.bfloat16).to(DEV)  # noqa: E731
        self.M, self.C, self.I = M, C, I
        self.residual, self.x, self.d_out, self.d_res = rand(M, C), rand(M, C, std=0.5), rand(M, C, std=1e-3), rand(M, C, std=1e-3)
        self.norm, self.w_up, self.w_down = rand(C, std=0.1) + 1, rand(2 * I, C, std=C ** -0.5), rand(C, I, std=I ** -0.5)
        self.c_up, self.c_down = Codes(2 * I, C, 0, 128).of(self.w_up), Codes(C, I, 0, 128).of(self.w_down)
        self.cy, self.ch, self.c_dout, self.c_dgu = Codes(M, C, 0, 1), Codes(M, I, 0, 1), Codes(M, C, 1, 1), Codes(M, 2 * I, 1, 1)
        self.res, self.rstd, self.h, self.gu, self.out = bf(M, C), f32(M), bf(M, I), bf(M, 2 * I), bf(M, C)
        self.dgu, self.h_again, self.dy, self.dx, self.dw_up, self.dw_down, self.dnorm = bf(M, 2 * I), bf(M, I), bf(M, C), bf(M, C), bf(2 * I, C), bf(C, I), f32(C)
        self.amax_h, self.amax_dgu, self.amax_dx, self.scale_dx = f32(1), f32(1), f32(1), f32(1)
        self.ws = u8(llmq.llmq_rmsnorm_bwd_workspace_bytes(M, C))

    def forward(self):
        llmq.llmq_rmsnorm_fwd_fp8_blocks(self.residual, self.x, self.norm, EPS, self.res, self.rstd, 0, self.cy.q, self.cy.s, self.cy.q_t, self.cy.s_t)
        llmq.llmq_fp8_gemm_blocks_swiglu_fwd(self.cy.q, self.cy.s, 0, self.c_up.q, self.c_up.s, 0, self.h, self.gu, self.amax_h)
        self.ch.of(self.h)
        llmq.llmq_fp8_gemm_blocks(self.ch.q, self.ch.s, 0, self.c_down.q, self.c_down.s, 0, self.out)

    def backward(self, accumulate):
        """h is not kept but comes once more from the gradient's kernel."""
        self.c_dout.of(self.d_out)
        llmq.llmq_fp8_gemm_blocks_swiglu_bwd(self.c_dout.q, self.c_dout.s, 1, self.c_down.q_t, self.c_down.s_t, 0, self.gu, self.dgu, self.h_again, self.amax_dgu)
        self.ch.of(self.h_again)
        llmq.llmq_fp8_gemm_blocks(self.c_dout.q_t, self.c_dout.s_t, 1, self.ch.q_t, self.ch.s_t, 0, self.dw_down, accumulate)
        self.c_dgu.of(self.dgu)
        llmq.llmq_fp8_gemm_blocks(self.c_dgu.q_t, self.c_dgu.s_t, 1, self.cy.q_t, self.cy.s_t, 0, self.dw_up, accumulate)
        llmq.llmq_fp8_gemm_blocks(self.c_dgu.q, self.c_dgu.s, 1, self.c_up.q_t, self.c_up.s_t, 0, self.dy)
        llmq.llmq_rmsnorm_bwd(self.dy, self.d_res, self.res, self.norm, self.rstd, self.dx, self.dnorm, accumulate, 1, self.amax_dx, self.scale_dx, self.ws)

    def step(self):
        for accumulate in (False, True):
            self.forward()
            self.backward(accumulate)

    def state(self):
        return [t.clone() for t in (self.res, self.rstd, self.cy.q, self.cy.q_t, self.cy.s, self.cy.s_t, self.h, self.gu, self.out, self.dgu, self.h_again, self.dy, self.dx, self.dw_up, self.dw_down, self.dnorm, self.amax_h,
                                    self.amax_dgu, self.amax_dx, self.scale_dx)]


def product(a, b):
    """(a b^T, what it may be off by before its rounding: 2^-11 of the sum of the products' magnitudes, that the matrix cores lose where they align 128 of them, and a binary32 addition a step)"""
    return a @ b.T, (2.0 ** -11 + -(-a.shape[1] // 128) * 2.0 ** -23) * (np.abs(a) @ np.abs(b).T)


def within(got, want, room, what):
    err = np.abs(f64(got) - want)
    assert (err <= room).all(), "%s: worst %g of the room" % (what, (err / np.maximum(room, 1e-300)).max())


@pytest.mark.parametrize("M,C,I", [(200, 384, 448), (20, 320, 1000), (333, 264, 136)])
def test_each_stage(M, C, I):
    b = Half(M, C, I, 1)
    b.forward()
    stream = (b.residual.float() + b.x.float()).to(torch.bfloat16)
    assert torch.equal(b.res, stream)
    r, w = f64(stream), f64(b.norm)
    rstd = 1 / np.sqrt((r * r).mean(1) + EPS)
    np.testing.assert_allclose(f64(b.rstd), rstd, rtol=2.0 ** -24 + C * 2.0 ** -52, atol=0)
    # codes of a value that may have been rounded the other way: half a step of BF16, 2^-17 of rstd, and half a step of E4M3, 2^-4, or, next to zero, half of its smallest step 2^-9 under the block's scale
    y = r * rstd[:, None] * w
    for transposed in (False, True):
        cy, want = b.cy.values(transposed), y.T if transposed else y
        scale = bc.scale_bytes(b.cy.s_t if transposed else b.cy.s, *want.shape).repeat(128, 1)[:, : want.shape[1]].astype(np.float64) - 127
        assert (np.abs(cy - want) <= (2.0 ** -4 + 2.0 ** -7) * np.abs(want) + 2.0 ** -10 * np.exp2(scale)).all()
    s, d = product(b.cy.values(), b.c_up.values())
    within(b.gu, s, d + 2.0 ** -8 * (np.abs(s) + d), "gate and up")
    g, u, eg, eu = s[:, :I], s[:, I:], d[:, :I], d[:, I:]
    silu = g / (1 + np.exp(-g))
    err = 1.1 * (np.abs(u) + eu) * eg + (np.abs(silu) + 1.1 * eg) * eu
    within(b.h, silu * u, err + (2.0 ** -8 + 2.0 ** -19 + 2.0 ** -24 * (np.abs(g) + eg)) * (np.abs(silu * u) + err) + 2.0 ** -118, "h")
    out, d = product(b.ch.values(), b.c_down.values())
    within(b.out, out, d + 2.0 ** -8 * (np.abs(out) + d), "down")
    assert b.amax_h.item() == b.h.abs().max().item()

    b.backward(False)
    dh, d = product(b.c_dout.values(), b.c_down.values(True))
    g, u = f64(b.gu[:, :I]), f64(b.gu[:, I:])
    sg = 1 / (1 + np.exp(-g))
    F, rel = sg * (1 + g * (1 - sg)), 2.0 ** -8 + 2.0 ** -19 + 2.0 ** -24 * np.abs(g)
    room = d * np.abs(u * F) + (np.abs(dh) + d) * np.abs(u) * sg * (1 + np.abs(g)) * (2.0 ** -19 + 2.0 ** -24 * np.abs(g))
    within(b.dgu[:, :I], dh * u * F, room + rel * (np.abs(dh * u * F) + room) + 2.0 ** -118, "gradient of the gates")
    room = d * np.abs(g * sg)
    within(b.dgu[:, I:], dh * g * sg, room + rel * (np.abs(dh * g * sg) + room) + 2.0 ** -118, "gradient of the ups")
    within(b.h_again, g * sg * u, rel * np.abs(g * sg * u) + 2.0 ** -118, "h once more")
    assert b.amax_dgu.item() == b.dgu.abs().max().item()
    for got, A, B, what in ((b.dw_down, b.c_dout.values(True), b.ch.values(True), "down weights"), (b.dw_up, b.c_dgu.values(True), b.cy.values(True), "up weights"),
                            (b.dy, b.c_dgu.values(), b.c_up.values(True), "input gradient")):
        want, d = product(A, B)
        within(got, want, d + 2.0 ** -8 * (np.abs(want) + d), what)
    n, dy = r * f64(b.rstd)[:, None], f64(b.dy)
    gw = dy * w
    mean = (gw * n).mean(1, keepdims=True)
    dx = f64(b.d_res) + f64(b.rstd)[:, None] * (gw - n * mean)
    size = np.abs(f64(b.d_res)) + f64(b.rstd)[:, None] * (np.abs(gw) + np.abs(n) * np.abs(gw * n).mean(1, keepdims=True))
    within(b.dx, dx, 2.0 ** -8 * np.abs(dx) + 2.0 ** -18 * size, "gradient of the norm")
    within(b.dnorm, (dy * n).sum(0), 2.0 ** -24 * (M // 64 + 40) * np.abs(dy * n).sum(0), "gradient of the norm's weights")
    assert b.amax_dx.item() == b.dx.abs().max().item()
    first = b.dw_up.clone(), b.dnorm.clone()
    b.backward(True)
    assert torch.allclose(b.dnorm, 2 * first[1], rtol=2.0 ** -22, atol=0)
    want, d = product(b.c_dgu.values(True), b.cy.values(True))
    want, d = want + f64(first[0]), d + 2.0 ** -24 * np.abs(want + f64(first[0]))
    within(b.dw_up, want, d + 2.0 ** -8 * (np.abs(want) + d), "added up weights")


def test_the_operators_that_are_joined_give_what_they_give_apart():
    """Norm (from its statistic) and quantizer; gate and up product.  h and the gradients differ by what is not rounded in between, half a step of BF16 of every factor."""
    b = Half(300, 512, 640, 3)
    b.forward()
    b.backward(False)
    M, C, I = b.M, b.C, b.I
    res, y, rstd, a = bf(M, C), bf(M, C), f32(M), f32(1)
    llmq.llmq_rmsnorm_fwd(b.residual, b.x, b.norm, EPS, res, y, rstd, 0, a, None, u8(llmq.llmq_rmsnorm_workspace_bytes(M)))
    assert ((rstd - b.rstd).abs() <= 2.0 ** -18 * rstd).all()                 # (sums in binary32)
    c = Codes(M, C, 0, 1).of((res.float() * b.rstd[:, None] * b.norm.float()).to(torch.bfloat16))
    assert all(torch.equal(p, q) for p, q in ((res, b.res), (c.q, b.cy.q), (c.s, b.cy.s), (c.q_t, b.cy.q_t), (c.s_t, b.cy.s_t)))
    gu, h = bf(M, 2 * I), bf(M, I)
    llmq.llmq_fp8_gemm_blocks(c.q, c.s, 0, b.c_up.q, b.c_up.s, 0, gu)
    room = product(c.values(), b.c_up.values())[1]
    assert (np.abs(f64(gu) - f64(b.gu)) <= 2 * room + 2.0 ** -7 * (np.abs(f64(gu)) + room)).all()
    ws = u8(llmq.llmq_swiglu_workspace_bytes(M, I))
    llmq.llmq_swiglu_fwd(gu, h, 0, f32(1), None, ws)
    g, u = np.abs(f64(gu[:, :I])), np.abs(f64(gu[:, I:]))
    eg, eu = room[:, :I] + 2.0 ** -8 * g, room[:, I:] + 2.0 ** -8 * u
    # twice: the gates and ups that either side starts from differ by at most that from the exact ones
    assert (np.abs(f64(h) - f64(b.h)) <= 2 * (1.1 * (u + eu) * eg + (g + 1.1 * eg) * eu) + 2.0 ** -6 * np.abs(f64(h)) + 2.0 ** -118).all()


def test_the_same_step_on_another_stream_and_from_a_graph():
    def eager(b):
        b.step()
        return b.state()

    def other_stream(b):
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            b.step()
        side.synchronize()
        return b.state()

    def replayed(b):
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                b.step()
        first = None
        for _ in range(4):
            for t in (b.res, b.h, b.gu, b.dgu, b.dx, b.dw_up, b.dnorm, b.amax_h, b.amax_dgu, b.amax_dx):
                t.fill_(3.0)                                                # what the step writes is not what is there
            graph.replay()
            torch.cuda.synchronize()
            state = b.state()
            first = first or state
            assert all(torch.equal(x, y) for x, y in zip(first, state))
            torch.zeros(1 << 20, device=DEV).normal_()                    # eager work in between
        return state

    for M in (150, 24):
        b = Half(M, 256, 384, 7)
        torch.cuda.synchronize()
        want = eager(b)
        for run in (other_stream, replayed):
            other = Half(M, 256, 384, 7)
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(want, run(other)))


def test_two_steps_at_once_on_their_own_streams():
    """Two blocks' steps side by side, each with its own buffers: what they give one after the other."""
    def run(together):
        halves, streams = [Half(M, 256, 384, k) for k, M in ((1, 150), (2, 24))], [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(3):
            for b, side in zip(halves, streams):
                with torch.cuda.stream(side if together else streams[0]):
                    b.step()
        torch.cuda.synchronize()
        return [t for b in halves for t in b.state()]

    assert all(torch.equal(a, b) for a, b in zip(run(False), run(True)))
