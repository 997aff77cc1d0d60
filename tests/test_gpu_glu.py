"""GPU parity: contractions of operands with block scales joined with a SwiGLU, against binary64.

Tolerances.  A sum is off by at most d = (2^-11 + steps 2^-23) S, S the sum of its products' magnitudes: the matrix cores align the 128 products of a K step to the largest (2^-12.3 of S was seen to be lost in
the plain contraction; twice that here) and the steps are added in binary32.  What the formulas make of that goes by their derivatives, |silu'| <= 1.1 and the factor F of dG below 1.1; the hardware's
exponential and reciprocal by 2^-20 + 2^-24 |g| of the sigmoid; four or five roundings in binary32, together below 2^-21; and a BF16 rounding by 2^-8 of the value (half of finfo.eps)."""
import numpy as np
import pytest
import torch

from paper_2512_15306_amd import llmq
from tests import blocks_common as bc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TINY = 2.0 ** -118


def operand(g, rows, T, fmt, std):
    """Codes, scale bytes and the values they stand for [rows, T] in binary64, on the GPU."""
    codes = (torch.randn(rows, T, generator=g) * 40).to(bc.FLOAT8[fmt])
    exponent = int(np.floor(np.log2(std / 40)))
    b = torch.randint(127 + exponent - 1, 127 + exponent + 2, (rows, bc.padded(T) // 128), generator=g).numpy()
    scale = torch.from_numpy(np.ldexp(1.0, b - 127)).repeat_interleave(128, 1)[:, :T]
    return codes.view(torch.uint8).to(DEV), bc.packed(b).to(DEV), (codes.to(torch.float64) * scale).to(DEV)


def empty(*shape):
    """Filled with rubbish, and a strip of it behind the last element."""
    n = int(np.prod(shape))
    t = torch.full((n + 64,), -7.0, device=DEV, dtype=torch.bfloat16)
    return t[:n].view(*shape), t[n:]


def product(A, B):
    """Sums and the bound of their error."""
    steps = -(-A.shape[1] // 128)
    return A @ B.t(), (2.0 ** -11 + steps * 2.0 ** -23) * (A.abs() @ B.abs().t())


def within(got, want, err, what):
    got = got.double()
    bad = ((got - want).abs() > err).nonzero()
    assert bad.shape[0] == 0, "%s: %d of %d out of tolerance, first %s got %r want %r bound %r" % (what, len(bad), want.numel(), bad[0].tolist(), *(float(t[tuple(bad[0])]) for t in (got, want, err)))


def forward(M, I, T, fmt, seed, keep=True):
    g = torch.Generator().manual_seed(seed)
    (a, sa, A), (w, sw, W) = operand(g, M, T, fmt, 1.0), operand(g, 2 * I, T, 0, 1.5 / np.sqrt(T))
    (h, strip), (gu, strip2) = empty(M, I), empty(M, 2 * I)
    amax = torch.full((1,), -1.0, device=DEV)
    llmq.llmq_fp8_gemm_blocks_swiglu_fwd(a, sa, fmt, w, sw, 0, h, gu if keep else None, amax)
    assert (strip == -7).all() and (strip2 == -7).all()
    s, d = product(A, W)
    x, u, dx, du = s[:, :I], s[:, I:], d[:, :I], d[:, I:]
    silu = x * torch.sigmoid(x)
    want = silu * u
    err = 1.1 * (u.abs() + du) * dx + (silu.abs() + 1.1 * dx) * du
    err = err + (2.0 ** -8 + 2.0 ** -19 + 2.0 ** -24 * (x.abs() + dx)) * (want.abs() + err) + TINY
    within(h, want, err, "h")
    if keep:
        within(gu, s, d + 2.0 ** -8 * (s.abs() + d), "gu")
    else:
        assert (gu == -7).all()
    check_amax(amax, h)
    return a, sa, w, sw, h, gu, amax


def check_amax(amax, t):
    am = torch.empty(1, device=DEV)
    llmq.llmq_amax_static(t, 0, am, None)
    assert torch.equal(amax, am)


def gradient(dh, d, x, u):
    """(want, err) of dG, dU, h from dh known within d."""
    sg = torch.sigmoid(x)
    F, s = sg * (1 + x * (1 - sg)), x * sg
    rel = 2.0 ** -8 + 2.0 ** -19 + 2.0 ** -24 * x.abs()
    dg, du, h = dh * u * F, dh * s, s * u
    eg = d * (u * F).abs() + (dh.abs() + d) * u.abs() * sg * (1 + x.abs()) * (2.0 ** -19 + 2.0 ** -24 * x.abs())
    eu = d * s.abs()
    return (dg, eg + rel * (dg.abs() + eg) + TINY), (du, eu + rel * (du.abs() + eu) + TINY), (h, rel * h.abs() + TINY)


def backward(M, I, T, fmt, seed, want_h=True, in_place=False):
    g = torch.Generator().manual_seed(seed)
    (a, sa, A), (b, sb, B) = operand(g, M, T, fmt, 1e-2), operand(g, I, T, 0, 0.5)
    kept = (torch.randn(M, 2 * I, generator=g) * 2).to(torch.bfloat16).to(DEV)
    gu, (dgu, strip), (h, strip2) = kept.clone(), empty(M, 2 * I), empty(M, I)
    if in_place:
        dgu = gu
    amax = torch.full((1,), -1.0, device=DEV)
    llmq.llmq_fp8_gemm_blocks_swiglu_bwd(a, sa, fmt, b, sb, 0, gu, dgu, h if want_h else None, amax)
    assert (strip == -7).all() and (strip2 == -7).all() and (in_place or torch.equal(gu, kept))
    (dg, eg), (du, eu), (y, ey) = gradient(*product(A, B), kept[:, :I].double(), kept[:, I:].double())
    within(dgu[:, :I], dg, eg, "dG")
    within(dgu[:, I:], du, eu, "dU")
    if want_h:
        within(h, y, ey, "h")
    else:
        assert (h == -7).all()
    check_amax(amax, dgu)
    return a, sa, b, sb, kept, dgu, h


FEW = [(1, 1, 16), (1, 16, 128), (7, 40, 100), (16, 100, 1000), (17, 333, 1111), (32, 512, 640), (16, 4096, 256), (31, 2050, 144), (3, 4608, 400), (2, 24, 4000)]
RAGGED = [(33, 1, 16), (40, 17, 100), (100, 100, 1000), (129, 65, 130), (200, 333, 256), (64, 96, 17), (300, 1000, 112), (257, 160, 2048), (1, 1000, 48), (513, 2720, 1000), (130, 992, 1024)]
WHOLE = [(128, 128, 128), (128, 64, 384), (256, 256, 1024), (384, 512, 128), (768, 1024, 256), (1024, 640, 512), (192, 128, 256)]


@pytest.mark.parametrize("M,I,T", FEW + RAGGED + WHOLE)
@pytest.mark.parametrize("fmt,keep", [(0, True), (1, False)])
def test_forward(M, I, T, fmt, keep):
    print("glu forward", M, I, T, fmt, keep, flush=True)
    forward(M, I, T, fmt, M + I + T, keep)


@pytest.mark.parametrize("M,I,T", FEW + RAGGED + WHOLE)
@pytest.mark.parametrize("fmt,h,in_place", [(0, True, False), (1, False, True)])
def test_backward(M, I, T, fmt, h, in_place):
    print("glu backward", M, I, T, fmt, h, in_place, flush=True)
    backward(M, I, T, fmt, M + I + T, h, in_place)


TILES = ["4x4", "3x4", "4x2", "2x4", "2x2"]


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("M,I,T", [(768, 512, 512), (768, 256, 128), (300, 320, 384), (450, 192, 1040), (257, 96, 144), (1000, 104, 272), (520, 2720, 272), (300, 320, 388), (450, 192, 1044), (257, 96, 20),
                                   (520, 2720, 1000), (1000, 104, 124), (200, 64, 252)])
def test_every_tile(monkeypatch, tile, M, I, T):
    """Whole tiles and guarded ones, with few K steps and more; sums in the order of the plain contraction: the same bytes in the kept GU."""
    print("glu tile", tile, M, I, T, flush=True)
    monkeypatch.setenv("LLMQ_GLU_TILE", tile)
    a, sa, w, sw, h, gu, _ = forward(M, I, T, 0, 5)
    c = torch.empty(M, 2 * I, device=DEV, dtype=torch.bfloat16)
    llmq.llmq_fp8_gemm_blocks(a, sa, 0, w, sw, 0, c)
    assert torch.equal(c, gu)
    alone = torch.empty_like(h)
    llmq.llmq_fp8_gemm_blocks_swiglu_fwd(a, sa, 0, w, sw, 0, alone)
    assert torch.equal(alone, h)
    a, sa, b, sb, kept, dgu, h = backward(M, I, T, 1, 6)
    again = torch.empty_like(dgu)
    llmq.llmq_fp8_gemm_blocks_swiglu_bwd(a, sa, 1, b, sb, 0, kept, again)
    assert torch.equal(again, dgu)


@pytest.mark.parametrize("slots", ["8", "64"])
@pytest.mark.parametrize("tile", ["4x4", "2x2"])
def test_many_rounds(monkeypatch, slots, tile):
    monkeypatch.setenv("LLMQ_GLU_TILE", tile)
    monkeypatch.setenv("LLMQ_GEMM_SLOTS", slots)
    monkeypatch.setenv("LLMQ_GEMM_TOUCH_NEXT", "1")
    forward(2048, 1024, 384, 0, 8)
    backward(2048, 1024, 384, 0, 9)


@pytest.mark.parametrize("M,I,T", [(100, 100, 1000), (70, 512, 512), (250, 37, 333)])
def test_few_rows_kernel_in_groups(monkeypatch, M, I, T):
    monkeypatch.setenv("LLMQ_GLU_FEW", "1")
    forward(M, I, T, 0, 3)
    backward(M, I, T, 0, 4)
    monkeypatch.setenv("LLMQ_GLU_FEW", "0")
    forward(20, I, T, 1, 3)
    backward(20, I, T, 1, 4)


@pytest.mark.parametrize("M,I,T", [(1, 16, 128), (16, 100, 1008), (17, 333, 1104), (32, 512, 640), (16, 5504, 272), (25, 4104, 4000), (130, 250, 2064), (17, 333, 1101), (2, 700, 4001), (450, 438, 223), (31, 96, 1404)])
@pytest.mark.parametrize("alone", ["0", "1"])
def test_few_rows_kernel_with_one_wave_and_four(monkeypatch, alone, M, I, T):
    print("glu few", alone, M, I, T, flush=True)
    monkeypatch.setenv("LLMQ_GLU_FEW", "1")
    monkeypatch.setenv("LLMQ_GLU_FEW_ALONE", alone)
    forward(M, I, T, 1, 3)
    backward(M, I, T, 0, 4)


@pytest.mark.parametrize("M", [20, 300])
def test_far_gates(M):
    """Gates far from zero on both sides: silu(g) is g or nearly nothing, never NaN."""
    I, T = 256, 256
    g = torch.Generator().manual_seed(1)
    (a, sa, A), (w, sw, W) = operand(g, M, T, 0, 1.0), operand(g, 2 * I, T, 0, 8.0)
    h, gu = torch.empty(M, I, device=DEV, dtype=torch.bfloat16), torch.empty(M, 2 * I, device=DEV, dtype=torch.bfloat16)
    llmq.llmq_fp8_gemm_blocks_swiglu_fwd(a, sa, 0, w, sw, 0, h, gu)
    x, u = gu[:, :I].double(), gu[:, I:].double()
    assert x.max() > 100 and x.min() < -100 and torch.isfinite(h).all()
    assert (h[x < -100] == 0).logical_or(h[x < -100].double().abs() < 2.0 ** -100).all()
    assert ((h.double() - x * u).abs() <= 2.0 ** -6 * (x * u).abs())[x > 20].all()
    dgu = torch.empty_like(gu)
    llmq.llmq_fp8_gemm_blocks_swiglu_bwd(a, sa, 0, w[:I].contiguous(), sw.view(2, -1)[:, :I].contiguous().view(-1), 0, gu, dgu)
    assert torch.isfinite(dgu).all() and (dgu[:, :I][x < -110].double().abs() < 2.0 ** -100).all()


@pytest.mark.parametrize("M,I,T", [(300, 96, 68), (300, 96, 1000), (513, 2720, 132), (20, 100, 332), (300, 100, 332), (300, 96, 130), (300, 100, 77), (140, 64, 255), (130, 34, 389), (513, 2720, 141), (7, 40, 1004), (33, 50, 517)])
@pytest.mark.parametrize("few,alone", [("0", "0"), ("1", "0"), ("1", "1")])
def test_what_lies_behind_a_row_does_not_count(monkeypatch, M, I, T, few, alone):
    """Rows that end inside a chunk of sixteen codes: the next row's first codes, and what lies behind the last row, are NaN."""
    print("glu behind rows", M, I, T, few, alone, flush=True)
    monkeypatch.setenv("LLMQ_GLU_FEW", few)
    monkeypatch.setenv("LLMQ_GLU_FEW_ALONE", alone)
    g = torch.Generator().manual_seed(T)
    (a, sa, A), (w, sw, W), (b, sb, B) = operand(g, M, T, 0, 1.0), operand(g, 2 * I, T, 0, 1.5 / np.sqrt(T)), operand(g, I, T, 0, 0.5)
    gu = (torch.randn(M, 2 * I, generator=g) * 2).to(torch.bfloat16).to(DEV)

    def run(a, w, b):
        h, kept, dgu = (torch.empty(M, n, device=DEV, dtype=torch.bfloat16) for n in (I, 2 * I, 2 * I))
        llmq.llmq_fp8_gemm_blocks_swiglu_fwd(a, sa, 0, w, sw, 0, h, kept)
        llmq.llmq_fp8_gemm_blocks_swiglu_bwd(a, sa, 0, b, sb, 0, gu, dgu)
        return h, kept, dgu

    def inside(t):
        """The tensor in the middle of one of NaNs"""
        out = torch.full((t.numel() + 8192,), 0x7F, device=DEV, dtype=torch.uint8)
        out[4096 : 4096 + t.numel()] = t.view(-1)
        return out[4096 : 4096 + t.numel()].view(t.shape)

    want = run(a, w, b)
    assert all(torch.equal(x, y) for x, y in zip(want, run(inside(a), inside(w), inside(b))))
    a2, w2, b2 = a.clone(), w.clone(), b.clone()
    a2[1::2, :16], w2[1::2, :16], b2[1::2, :16] = 0x7F, 0x7F, 0xFF
    h, kept, dgu = run(a2, w2, b2)
    odd = torch.arange(2 * I) % 2 == 1                       # rows of W; I is even, so its ups' too
    assert torch.isnan(kept[1::2]).all() and torch.isnan(kept[:, odd]).all() and torch.isnan(h[1::2]).all()
    assert torch.equal(kept[::2, ~odd], want[1][::2, ~odd]) and torch.equal(h[::2, ::2], want[0][::2, ::2])
    assert torch.isnan(dgu[1::2]).all() and torch.isnan(dgu[:, odd]).all() and torch.equal(dgu[::2, ~odd], want[2][::2, ~odd])


@pytest.mark.parametrize("M", [20, 300])
def test_rows_that_are_not_numbers(M):
    """A block scale of 255 makes its own row NaN and no other."""
    I, T = 100, 300
    a, sa, w, sw, h, gu, _ = forward(M, I, T, 0, 2)
    bad = sa.clone()
    bad[int(bc.scale_places(M, 3)[5, 1])] = 255
    h2, gu2 = torch.empty_like(h), torch.empty_like(gu)
    llmq.llmq_fp8_gemm_blocks_swiglu_fwd(a, bad, 0, w, sw, 0, h2, gu2)
    others = [r for r in range(M) if r != 5]
    assert torch.isnan(h2[5]).all() and torch.isnan(gu2[5]).all() and torch.equal(h2[others], h[others]) and torch.equal(gu2[others], gu[others])
    a, sa, b, sb, kept, dgu, _ = backward(M, I, T, 0, 3)
    bad = sb.clone()
    bad[int(bc.scale_places(I, 3)[7, 2])] = 255
    d2 = torch.empty_like(dgu)
    llmq.llmq_fp8_gemm_blocks_swiglu_bwd(a, sa, 0, b, bad, 0, kept, d2)
    others = [c for c in range(2 * I) if c % I != 7]
    assert torch.isnan(d2[:, [7, I + 7]]).all() and torch.equal(d2[:, others], dgu[:, others])


def test_the_gradient_of_the_forward_formula():
    """gradient() above against differences of the forward formula, in binary64."""
    g = torch.Generator().manual_seed(4)
    x, u, dh = (torch.randn(50, 60, generator=g, dtype=torch.float64) * s for s in (3.0, 1.0, 1.0))
    (dg, _), (du, _), (h, _) = gradient(dh, torch.zeros_like(dh), x, u)
    f = lambda x, u: (x * torch.sigmoid(x) * u * dh).sum()  # noqa: E731
    assert torch.allclose(h, x * torch.sigmoid(x) * u)
    for _ in range(10):
        d, e = torch.randn(50, 60, generator=g, dtype=torch.float64), 1e-5
        assert abs((f(x + e * d, u) - f(x - e * d, u)) / (2 * e) - (dg * d).sum()) <= 1e-6 * (dg * d).abs().sum()
        assert abs((f(x, u + e * d) - f(x, u - e * d)) / (2 * e) - (du * d).sum()) <= 1e-6 * (du * d).abs().sum()


def test_captured_calls_on_a_stream_of_their_own():
    M, I, T = 200, 224, 640
    a, sa, w, sw, h, gu, amax = forward(M, I, T, 0, 2)
    b, sb, _ = operand(torch.Generator().manual_seed(8), I, T, 0, 0.5)
    dgu, h2 = torch.empty_like(gu), torch.empty_like(h)

    def step():
        llmq.llmq_fp8_gemm_blocks_swiglu_fwd(a, sa, 0, w, sw, 0, h, gu, amax)
        llmq.llmq_fp8_gemm_blocks_swiglu_bwd(a, sa, 0, b, sb, 0, gu, dgu, h2)

    outs = (h, gu, amax, dgu, h2)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for k in range(4):
        a.copy_(operand(torch.Generator().manual_seed(20 + k), M, T, 0, 1.0)[0])
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        for t in outs:
            t.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, outs))
