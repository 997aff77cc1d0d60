"""GPU parity: residual RMSNorm out as FP8 with block scales, and its gradient, against binary64 on the CPU.

Tolerances.  A BF16 rounding is off by at most 2^-8 of the value (half of finfo.eps), a binary32 one by 2^-24.
  rstd   sums in binary64, one rounding: 2^-24 (and C 2^-52 of the sums').
  y      from the rstd that was returned: two products and a rounding: 2^-8 + 2^-22.
  codes  from the y that was returned: exact.
  dx     mean(g n) has 8 VPL <= 64 terms in a lane's chain (C / 512 in rows beyond 16384), 6 steps of the wave and 8 waves, and three roundings a term; the result four more, and BF16's.
  dw     at most ceil(M / 64) rows in a lane's chain, 8 groups of rows, 16 rows of sums and 5 steps pairwise, and two roundings a term."""
import numpy as np
import pytest
import torch

from paper_2512_15306_amd import llmq, synth
from tests import blocks_common as bc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6
SHAPES = [(1, 1), (3, 100), (33, 17), (5, 264), (1, 3584), (130, 1024), (129, 257), (6, 8200), (2, 16392), (3, 16401), (40, 8192), (300, 384), (70, 2730), (530, 2304), (517, 2051), (515, 6152)]


def bf16(g, *shape, std=1.0):
    return (torch.randn(*shape, generator=g) * std).to(torch.bfloat16)


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def empty(*shape, dtype=torch.bfloat16):
    """Filled with rubbish."""
    return torch.full(shape, 0xAA, device=DEV, dtype=dtype) if dtype == torch.uint8 else torch.full(shape, -7.0, device=DEV, dtype=dtype)


def inputs(M, C, seed, add=True):
    g = torch.Generator().manual_seed(seed)
    res = bf16(g, M, C, std=1.3) * torch.exp(torch.randn(M, 1, generator=g)).to(torch.bfloat16)
    return res, bf16(g, M, C, std=0.4) if add else None, (1.0 + 0.2 * torch.randn(C, generator=g)).to(torch.bfloat16)


def forward(res, x, w, fmt, rows=True, cols=True, y=True, eps=EPS, in_place=False):
    M, C = res.shape
    r = res.to(DEV).clone()
    out = {"res": (r if in_place else empty(M, C)) if x is not None else None, "rstd": empty(M, dtype=torch.float32), "y": empty(M, C) if y else None, "q": None, "s": None, "qt": None, "st": None}
    if rows:
        out["q"], out["s"] = empty(M, C, dtype=torch.uint8), empty(llmq.llmq_block_scales_bytes(M, C), dtype=torch.uint8)
    if cols:
        out["qt"], out["st"] = empty(C, M, dtype=torch.uint8), empty(llmq.llmq_block_scales_bytes(C, M), dtype=torch.uint8)
    llmq.llmq_rmsnorm_fwd_fp8_blocks(r, x.to(DEV) if x is not None else None, w.to(DEV), eps, out["res"], out["rstd"], fmt, out["q"], out["s"], out["qt"], out["st"], out["y"])
    return out


def check_codes(y, q, s, fmt):
    rows, cols = y.shape
    codes, b = bc.quantize(y, fmt, 1)
    np.testing.assert_array_equal(bc.scale_bytes(s, rows, cols), b)
    np.testing.assert_array_equal(bc.decode(q, fmt), codes)
    spare = np.ones(s.numel(), dtype=bool)                          # bytes of rows that do not exist are written too
    spare[bc.scale_places(rows, bc.padded(cols) // 128)] = False
    assert (s.cpu().numpy()[spare] != 0xAA).all()


@pytest.mark.parametrize("M,C", SHAPES)
@pytest.mark.parametrize("rows,cols,add,fmt", [(True, False, True, 0), (True, True, True, 1), (False, True, False, 0), (True, False, False, 1)])
def test_forward(M, C, rows, cols, add, fmt):
    print("norm forward", M, C, rows, cols, add, fmt, flush=True)
    res, x, w = inputs(M, C, 7 * M + C, add)
    out = forward(res, x, w, fmt, rows, cols)
    stream = (res.float() + x.float()).to(torch.bfloat16) if add else res
    if add:
        assert torch.equal(out["res"].cpu(), stream)
    r = f64(stream)
    rstd = 1 / np.sqrt((r * r).mean(1) + EPS)
    np.testing.assert_allclose(f64(out["rstd"]), rstd, rtol=2.0 ** -24 + C * 2.0 ** -52, atol=0)
    y = r * f64(out["rstd"])[:, None] * f64(w)
    assert (np.abs(f64(out["y"]) - y) <= (2.0 ** -8 + 2.0 ** -22) * np.abs(y) + 2.0 ** -133).all()
    if rows:
        check_codes(out["y"], out["q"], out["s"], fmt)
    if cols:
        check_codes(out["y"].t().contiguous(), out["qt"], out["st"], fmt)


@pytest.mark.parametrize("M,C", SHAPES)
def test_forward_has_the_bytes_of_the_norm_and_the_quantizer(M, C):
    """The sum, y and its codes; the plain norm's own statistic has sums in binary32."""
    res, x, w = inputs(M, C, M + C)
    r, y, rstd, a = empty(M, C), empty(M, C), empty(M, dtype=torch.float32), empty(1, dtype=torch.float32)
    ws = torch.empty(llmq.llmq_rmsnorm_workspace_bytes(M), device=DEV, dtype=torch.uint8)
    llmq.llmq_rmsnorm_fwd(res.to(DEV), x.to(DEV), w.to(DEV), EPS, r, y, rstd, 0, a, None, ws)
    for cols in (False, True):
        out = forward(res, x, w, 0, cols=cols, y=cols, in_place=not cols)
        # 2^-17: at most 100 roundings behind one another (64 elements a lane, or C / 64 of wide rows, the wave, four waves), the rest four, half of it in the root
        assert torch.equal(out["res"], r) and ((out["rstd"] - rstd).abs() <= 2.0 ** -24 * (max(64, C // 64) + 48) / 2 * rstd).all()
        y = (out["res"].float() * out["rstd"][:, None] * w.to(DEV).float()).to(torch.bfloat16)
        q, s = empty(M, C, dtype=torch.uint8), empty(llmq.llmq_block_scales_bytes(M, C), dtype=torch.uint8)
        qt, st = empty(C, M, dtype=torch.uint8), empty(llmq.llmq_block_scales_bytes(C, M), dtype=torch.uint8)
        llmq.llmq_quantize_fp8_blocks(y, 0, 1, q, s, qt, st)
        assert torch.equal(out["q"], q) and torch.equal(out["s"], s)
        if cols:
            assert torch.equal(out["y"], y) and torch.equal(out["qt"], qt) and torch.equal(out["st"], st)


@pytest.mark.parametrize("M,C", [(1, 2304), (130, 4096), (257, 2051), (2100, 2176), (2049, 8192), (3, 16384)])
@pytest.mark.parametrize("fmt", [0, 1])
def test_every_kernel_of_the_forward_pass_gives_the_same_bytes(monkeypatch, M, C, fmt):
    res, x, w = inputs(M, C, 11)
    want = None
    for kernel in ("1", "2"):
        for one in ("0", "1"):
            print("norm kernel", kernel, one, M, C, fmt, flush=True)
            monkeypatch.setenv("LLMQ_NORM_KERNEL", kernel)
            monkeypatch.setenv("LLMQ_NORM_ONE", one)
            out = forward(res, x, w, fmt, cols=False)
            if want is None:
                want = out
                check_codes(out["y"], out["q"], out["s"], fmt)
            assert all(torch.equal(want[k], out[k]) for k in ("res", "rstd", "y", "q", "s"))


@pytest.mark.parametrize("C", [200, 1024, 4096])
def test_forward_rows_that_are_not_numbers(C):
    """An Inf or NaN marks its own row's blocks with 255 and leaves the other rows' bytes; rows of zeros have codes of zero, also where eps = 0 makes NaN of them."""
    res, x, w = inputs(140, C, 3)
    clean = forward(res, x, w, 0, cols=False)
    res[5, 7], res[130, C - 1] = float("inf"), float("nan")
    res[9], x[9] = 0, 0
    out = forward(res, x, w, 0, cols=False)
    b, codes = bc.scale_bytes(out["s"], 140, C), bc.decode(out["q"], 0)
    assert (b[130] == 255).all() and b[5, 0] == 255 and (b[9] == 127).all() and (codes[9] == 0).all()
    others = [r for r in range(140) if r not in (5, 9, 130)]
    np.testing.assert_array_equal(b[others], bc.scale_bytes(clean["s"], 140, C)[others])
    np.testing.assert_array_equal(codes[others], bc.decode(clean["q"], 0)[others])
    out = forward(res, x, w, 0, eps=0.0)
    assert (bc.scale_bytes(out["s"], 140, C)[9] == 255).all() and torch.isnan(out["y"][9]).all()
    np.testing.assert_array_equal(bc.scale_bytes(out["s"], 140, C)[[0, 139]], bc.scale_bytes(forward(res, x, w, 0, eps=0.0, cols=False)["s"], 140, C)[[0, 139]])


def grad_inputs(M, C, seed, dres=True):
    res, _, w = inputs(M, C, seed, False)
    g = torch.Generator().manual_seed(seed + 1)
    r = f64(res)
    return {"dy": bf16(g, M, C, std=1e-2), "dres": bf16(g, M, C, std=1e-2) if dres else None, "res": res, "w": w, "rstd": torch.from_numpy(1 / np.sqrt((r * r).mean(1) + EPS)).float()}


def backward(i, want_dw=True, want_amax=True, dw=None, fmt=1, alias=None):
    M, C = i["res"].shape
    d = {k: v.to(DEV).clone() if v is not None else None for k, v in i.items()}
    dx = d[alias] if alias else empty(M, C)
    acc = dw is not None
    dw = dw if acc else empty(C, dtype=torch.float32) if want_dw else None
    a, s = (empty(1, dtype=torch.float32), empty(1, dtype=torch.float32)) if want_amax else (None, None)
    ws = torch.full((llmq.llmq_rmsnorm_bwd_workspace_bytes(M, C),), 0xFF, device=DEV, dtype=torch.uint8) if want_dw or want_amax else None
    llmq.llmq_rmsnorm_bwd(d["dy"], d["dres"], d["res"], d["w"], d["rstd"], dx, dw, acc, fmt, a, s, ws)
    return dx, dw, a, s


def plain_backward(i):
    """(dx, bound of its error, dw, bound of its error) in binary64."""
    dy, r, w, res = f64(i["dy"]), f64(i["rstd"])[:, None], f64(i["w"]), f64(i["res"])
    M, C = res.shape
    n, g = res * r, dy * w
    mean = (g * n).mean(1, keepdims=True)
    dx = r * (g - n * mean)
    chain = (64 if C <= 16384 else C // 512 + 1) + 6 + 8 + 3 + 1
    err = 2.0 ** -24 * r * (np.abs(n) * chain * np.abs(g * n).mean(1, keepdims=True) + 4 * (np.abs(g) + np.abs(n * mean)))
    if i["dres"] is not None:
        dx = dx + f64(i["dres"])
        err = err + 2.0 ** -24 * np.abs(dx)
    return dx, 2.0 ** -8 * np.abs(dx) + (1 + 2.0 ** -8) * err + 2.0 ** -133, (dy * n).sum(0), 2.0 ** -24 * (-(-M // 64) + 8 + 16 + 5 + 2) * np.abs(dy * n).sum(0)


@pytest.mark.parametrize("M,C", [(1, 1), (3, 100), (33, 17), (5, 264), (1, 3584), (130, 1024), (700, 512), (4100, 600), (4099, 2048), (6, 8200), (2, 16384), (3, 16401), (70, 20000), (300, 384), (70, 2730),
                                 (1030, 2304), (517, 2051), (515, 6152), (1025, 8192)])
@pytest.mark.parametrize("dres", [True, False])
def test_backward(M, C, dres):
    print("norm backward", M, C, dres, flush=True)
    i = grad_inputs(M, C, M + C, dres)
    dx, dw, a, s = backward(i)
    want, err, want_dw, err_dw = plain_backward(i)
    assert (np.abs(f64(dx) - want) <= err).all()
    assert (np.abs(f64(dw) - want_dw) <= err_dw).all()
    am, sc = empty(1, dtype=torch.float32), empty(1, dtype=torch.float32)
    llmq.llmq_amax_static(dx, 1, am, sc)
    assert torch.equal(a, am) and torch.equal(s, sc)
    # what is not wanted leaves the rest as it is; the sums are the same from run to run, and added to what is there
    for kw in (dict(want_dw=False), dict(want_amax=False), dict(want_dw=False, want_amax=False), dict(alias="dy")) + ((dict(alias="dres"),) if dres else ()):
        other = backward(i, **kw)
        assert torch.equal(other[0], dx), kw
        assert other[1] is None or torch.equal(other[1], dw), kw
    start = torch.arange(C, device=DEV, dtype=torch.float32)
    assert torch.equal(backward(i, dw=start.clone())[1], start + dw)


def test_backward_is_the_gradient():
    """The formula of plain_backward against differences of the forward formula, and the kernel's mean output over the same inputs against it."""
    i = grad_inputs(7, 96, 11, False)
    dy, res, w = f64(i["dy"]), f64(i["res"]), f64(i["w"])
    i["rstd"] = torch.from_numpy(1 / np.sqrt((res * res).mean(1) + EPS))          # (binary64 here)
    loss = lambda x, v: (dy * x / np.sqrt((x * x).mean(1, keepdims=True) + EPS) * v).sum()  # noqa: E731
    dx, _, dw, _ = plain_backward(i)
    rng = np.random.default_rng(5)
    for _ in range(20):
        d, h = rng.standard_normal(res.shape), 1e-5
        assert abs((loss(res + h * d, w) - loss(res - h * d, w)) / (2 * h) - (dx * d).sum()) <= 1e-6 * np.abs(dx * d).sum()
        d = rng.standard_normal(w.shape)
        assert abs((loss(res, w + h * d) - loss(res, w - h * d)) / (2 * h) - (dw * d).sum()) <= 1e-6 * np.abs(dw * d).sum()


@pytest.mark.parametrize("C", [264, 2730, 5120])
def test_backward_keeps_bad_rows_to_themselves(C):
    i = grad_inputs(200, C, 4)
    clean = backward(i)[0]
    i["dy"][17, 3], i["res"][130, C - 1] = float("nan"), float("inf")
    dx = backward(i)[0]
    good = [r for r in range(200) if r not in (17, 130)]
    assert torch.equal(dx[good], clean[good]) and torch.isnan(dx[17]).any() and not torch.isfinite(dx[130]).all()


def test_nothing_beside_the_outputs_is_written():
    M, C = 131, 2731
    i = grad_inputs(M, C, 6)
    d = {k: v.to(DEV) for k, v in i.items()}
    big, bigw = empty(M * C + 64), empty(C + 64, dtype=torch.float32)
    llmq.llmq_rmsnorm_bwd(d["dy"], d["dres"], d["res"], d["w"], d["rstd"], big[: M * C].view(M, C), bigw[:C], False, 0, None, None,
                          torch.empty(llmq.llmq_rmsnorm_bwd_workspace_bytes(M, C), device=DEV, dtype=torch.uint8))
    assert (big[M * C:] == -7).all() and (bigw[C:] == -7).all()
    q, qt, rs, y = empty(M * C + 64, dtype=torch.uint8), empty(M * C + 64, dtype=torch.uint8), empty(M + 64, dtype=torch.float32), empty(M * C + 64)
    n, nt = llmq.llmq_block_scales_bytes(M, C), llmq.llmq_block_scales_bytes(C, M)
    s, st = empty(n + 64, dtype=torch.uint8), empty(nt + 64, dtype=torch.uint8)
    for both in (True, False):
        llmq.llmq_rmsnorm_fwd_fp8_blocks(d["res"], None, d["w"], EPS, None, rs[:M], 0, q[: M * C].view(M, C), s[:n], qt[: M * C].view(C, M) if both else None, st[:nt] if both else None, y[: M * C].view(M, C))
        assert all((t[k:] == t[-1]).all() and float(t[-1]) in (-7.0, 170.0) for t, k in ((q, M * C), (qt, M * C), (s, n), (st, nt), (rs, M), (y, M * C)))


def test_captured_calls_on_a_stream_of_their_own():
    M, C = 300, 1000
    i = grad_inputs(M, C, 9)
    d = {k: v.to(DEV) for k, v in i.items()}
    q, s, rs, r2 = empty(M, C, dtype=torch.uint8), empty(llmq.llmq_block_scales_bytes(M, C), dtype=torch.uint8), empty(M, dtype=torch.float32), empty(M, C)
    qt, st = empty(C, M, dtype=torch.uint8), empty(llmq.llmq_block_scales_bytes(C, M), dtype=torch.uint8)
    dx, dw = empty(M, C), empty(C, dtype=torch.float32)
    ws = torch.empty(llmq.llmq_rmsnorm_bwd_workspace_bytes(M, C), device=DEV, dtype=torch.uint8)

    def step():
        llmq.llmq_rmsnorm_fwd_fp8_blocks(d["res"], d["dres"], d["w"], EPS, r2, rs, 0, q, s, qt, st)
        llmq.llmq_rmsnorm_bwd(d["dy"], d["dres"], r2, d["w"], rs, dx, dw, False, 0, None, None, ws)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for k in range(4):
        d["res"].copy_(inputs(M, C, 20 + k, False)[0])
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (q, s, qt, st, rs, r2, dx, dw)]
        for t in (q, s, qt, st, rs, r2, dx, dw):
            t.fill_(1)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (q, s, qt, st, rs, r2, dx, dw)))
