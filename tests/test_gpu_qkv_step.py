"""The operators around the linears in a row, as a training step of a QKV projection uses them: block-scaled forward product, query and key norms with the rotation, their
gradient, block-scaled input and weight gradients added up over two micro-steps, an AdamW step, and the next step on the new weights.  Every stage is checked on what the stage before
it left; then the same step on another stream and from a graph gives the same bytes."""
import numpy as np
import pytest
import torch

from paper_2512_15306_amd import llmq
from tests import adamw_common as ac
from tests import blocks_common as bc
from tests import qk_common as qc

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


class Step:
    def __init__(self, M, K, Hq, Hkv, D, seed):
        g = torch.Generator().manual_seed(seed)
        rand = lambda *n, std=1.0: torch.randn(*n, generator=g).mul(std).to(torch.bfloat16).to(DEV)  # noqa: E731
        self.M, self.K, self.Hq, self.Hkv, self.D, self.N = M, K, Hq, Hkv, D, (Hq + 2 * Hkv) * D
        self.x, self.dq, self.dk, self.dv = rand(M, K), rand(M, Hq * D, std=1e-3), rand(M, Hkv * D, std=1e-3), rand(M, Hkv * D, std=1e-3)
        self.master = torch.randn(self.N, K, generator=g).mul(0.02).to(DEV)
        self.w = self.master.to(torch.bfloat16)
        self.wq, self.wk = rand(D, std=0.1) + 1, rand(D, std=0.1) + 1
        self.positions, self.inv_freq = torch.arange(M, device=DEV) % 97, 10000.0 ** (-torch.arange(0, D, 2, device=DEV, dtype=torch.float64) / D)
        self.cx, self.cw, self.cd = Codes(M, K, 0, 1), Codes(self.N, K, 0, 128), Codes(M, self.N, 1, 1)
        self.qkv, self.q, self.k, self.rstd = bf(M, self.N), bf(M, Hq * D), bf(M, Hkv * D), f32(M, Hq + Hkv)
        self.dqkv, self.dwq, self.dwk, self.amax, self.scale = bf(M, self.N), f32(D), f32(D), f32(1), f32(1)
        self.ws = u8(llmq.llmq_qk_norm_rope_workspace_bytes(M, Hq, Hkv, D))
        self.dx, self.dw, self.amax_w = bf(M, K), bf(self.N, K), f32(1)
        n = self.N * K
        self.m, self.v, self.ms, self.vs = u8(n), u8(n), u8((n + 127) // 128) + 127, u8((n + 127) // 128) + 127
        self.mq, self.vq, self.mk, self.vk = f32(D), f32(D), f32(D), f32(D)
        self.hyper = llmq.llmq_adamw_hyper(1, 1e-3, 0.9, 0.95, 1e-8, 0.1, 3).to(DEV)
        T = llmq.AdamWTensor
        self.plan = llmq.llmq_adamw_plan([T(self.w, self.master, self.dw, self.m, self.v, self.ms, self.vs, 0, amax=self.amax_w),
                                          T(self.wq, None, self.dwq, self.mq, self.vq, first_counter=n, decay=False, stochastic=True),
                                          T(self.wk, None, self.dwk, self.mk, self.vk, first_counter=n + D, decay=False)])

    def micro_step(self, accumulate):
        llmq.llmq_fp8_gemm_blocks(self.cx.of(self.x).q, self.cx.s, 0, self.cw.of(self.w).q, self.cw.s, 0, self.qkv)
        llmq.llmq_qk_norm_rope_fwd(self.qkv, self.Hq, self.Hkv, self.D, self.wq, self.wk, EPS, self.positions, self.inv_freq, False, self.q, self.k, self.rstd)
        llmq.llmq_qk_norm_rope_bwd(self.dq, self.dk, self.dv, self.qkv, self.Hq, self.Hkv, self.D, self.wq, self.wk, self.rstd, self.positions, self.inv_freq, False, self.dqkv, self.dwq, self.dwk,
                                   accumulate, llmq.E5M2, self.amax, self.scale, self.ws)
        self.cd.of(self.dqkv)
        llmq.llmq_fp8_gemm_blocks(self.cd.q, self.cd.s, 1, self.cw.q_t, self.cw.s_t, 0, self.dx)
        llmq.llmq_fp8_gemm_blocks(self.cd.q_t, self.cd.s_t, 1, self.cx.q_t, self.cx.s_t, 0, self.dw, accumulate)

    def step(self):
        self.micro_step(False)
        self.micro_step(True)
        llmq.llmq_adamw_step(self.plan, self.hyper)

    def state(self):
        return [t.clone() for t in (self.w, self.master, self.m, self.v, self.ms, self.vs, self.wq, self.wk, self.qkv, self.q, self.k, self.dqkv, self.dx, self.dw, self.dwq, self.dwk, self.amax, self.amax_w)]


def product(a, b):
    """(a b^T, the sums of the products' magnitudes)"""
    return a @ b.T, np.abs(a) @ np.abs(b).T


def within(got, want, room, what):
    err = np.abs(f64(got) - want)
    assert (err <= room).all(), "%s: worst %g of the room" % (what, (err / np.maximum(room, 1e-300)).max())


def test_each_stage_of_a_step():
    s = Step(200, 384, 4, 2, 64, 1)
    s.micro_step(False)
    x, w, d = s.cx.values(), s.cw.values(), s.cd.values()
    for codes, t in ((s.cx, s.x), (s.cw, s.w), (s.cd, s.dqkv)):
        for transposed in (False, True):
            want, b = bc.quantize(t.t().contiguous() if transposed else t, codes.fmt, codes.block_rows)
            assert np.array_equal(codes.values(transposed), bc.values(want, b))
    y, S = product(x, w)
    within(s.qkv, y, 2.0 ** -7 * S, "forward")
    # the heads, with the bounds of the operator's own tests
    H, D = 6, 64
    angle, weights = qc.angles(s.positions.cpu().numpy(), f64(s.inv_freq)), np.concatenate([np.tile(f64(s.wq), (4, 1)), np.tile(f64(s.wk), (2, 1))])
    heads = f64(s.qkv)[:, : H * D].reshape(200, H, D)
    y, r, n = qc.forward(heads, weights, EPS, angle, D, False)
    within(torch.cat([s.q, s.k], 1), y.reshape(200, -1), (2.0 ** -8 * np.abs(y) + 2.0 ** -19 * qc.of_pairs(n, D, False)).reshape(200, -1), "heads")
    r = f64(s.rstd)
    dy = np.concatenate([f64(s.dq), f64(s.dk)], 1).reshape(200, H, D)
    dx, dw, _ = qc.backward(dy, heads, weights, r, angle, D, False)
    size, nn = qc.of_pairs(dy, D, False) * np.abs(weights), np.abs(heads * r[..., None])
    size = r[..., None] * (size + nn * (size * nn).mean(-1, keepdims=True))
    within(s.dqkv[:, : H * D], dx.reshape(200, -1), (2.0 ** -8 * np.abs(dx) + 2.0 ** -18 * size).reshape(200, -1), "gradient of the heads")
    assert torch.equal(s.dqkv[:, H * D :], s.dv) and s.amax.item() == s.dqkv.abs().max().item()
    within(s.dwq, dw[:, :4].sum((0, 1)), 2.0 ** -12 * (np.abs(dw[:, :4]).sum((0, 1)) + 1e-30), "gradient of a norm weight")
    y, S = product(d, s.cw.values(True))
    within(s.dx, y, 2.0 ** -7 * S, "input gradient")
    y, S = product(s.cd.values(True), s.cx.values(True))
    within(s.dw, y, 2.0 ** -7 * S, "weight gradient")
    first = s.dw.clone(), s.dwq.clone()
    s.micro_step(True)
    within(s.dw, f64(first[0]) + y, 2.0 ** -7 * (S + np.abs(f64(first[0]))), "added weight gradient")
    assert torch.allclose(s.dwq, 2 * first[1], rtol=2.0 ** -22, atol=0)
    state = ac.State(s.w.view(torch.int16).cpu().numpy().view(np.uint16).ravel(), s.master.cpu().numpy().ravel(), s.m.cpu().numpy(), s.v.cpu().numpy(), s.ms.cpu().numpy(), s.vs.cpu().numpy())
    want = ac.step_as_rounded(state, s.dw.float().cpu().numpy().ravel(), 1, 1e-3, 0.9, 0.95, 1e-8, 0.1, seed=3)
    llmq.llmq_adamw_step(s.plan, s.hyper)
    for got, exp in ((s.master, want.master), (s.m, want.m), (s.v, want.v), (s.ms, want.m_scale), (s.vs, want.v_scale)):
        assert np.array_equal(got.cpu().numpy().ravel(), exp.astype(got.cpu().numpy().dtype))
    # the absmax the step left is the scale a per-tensor quantization of the new weights starts from
    a, sc, sc2 = f32(1), f32(1), f32(1)
    llmq.llmq_amax(s.w, 0, a, sc, u8(llmq.llmq_amax_workspace_bytes()))
    llmq.llmq_scale_from_amax(s.amax_w, 0, sc2)
    assert torch.equal(sc, sc2)


def test_the_same_step_on_another_stream_and_from_a_graph():
    def steps(run):
        s = Step(130, 256, 2, 1, 128, 7)
        torch.cuda.synchronize()
        out = []
        run(s, out)
        return out

    def eager(s, out):
        for t in range(1, 5):
            s.hyper.copy_(llmq.llmq_adamw_hyper(t, 1e-3, 0.9, 0.95, 1e-8, 0.1, 3))
            s.step()
            out.append(s.state())

    def other_stream(s, out):
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            eager(s, out)
        side.synchronize()

    def replayed(s, out):
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                s.step()
        for t in range(1, 5):
            s.hyper.copy_(llmq.llmq_adamw_hyper(t, 1e-3, 0.9, 0.95, 1e-8, 0.1, 3))
            graph.replay()
            torch.cuda.synchronize()
            out.append(s.state())
            torch.zeros(1 << 20, device=DEV).normal_()                # eager work in between

    want = steps(eager)
    for run in (other_stream, replayed):
        for a, b in zip(want, steps(run)):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
    # weights have moved every step
    assert not any(torch.equal(a[1], b[1]) for a, b in zip(want, want[1:]))


def test_two_steps_at_once_on_their_own_streams():
    """Two layers' steps side by side, each with its own buffers: what they give one after the other."""
    def run(together):
        layers, streams = [Step(150, 256, 2, 1, 128, k) for k in (1, 2)], [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(3):
            for s, side in zip(layers, streams):
                with torch.cuda.stream(side if together else streams[0]):
                    s.step()
        torch.cuda.synchronize()
        return [t for s in layers for t in s.state()]

    assert all(torch.equal(a, b) for a, b in zip(run(False), run(True)))
