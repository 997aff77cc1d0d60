"""FP8 with a scale for each block of 128 on the GPU: the quantizer bit for bit, the contraction against binary64."""
import numpy as np
import pytest
import torch

from paper_2512_15306_amd import llmq
from tests import blocks_common as bc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def tensor(rows, cols, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(spread * torch.randn(rows, 1, generator=g)) * torch.exp(spread * torch.randn(1, cols, generator=g))
    return x.to(torch.bfloat16)


def run_quantize(x, fmt, block_rows, copies="both"):
    rows, cols = x.shape
    u8 = lambda *n: torch.full(n, 0xAB, device=DEV, dtype=torch.uint8)  # noqa: E731
    q, s = (u8(rows, cols), u8(llmq.llmq_block_scales_bytes(rows, cols))) if copies != "columns" else (None, None)
    qt, st = (u8(cols, rows), u8(llmq.llmq_block_scales_bytes(cols, rows))) if copies != "rows" else (None, None)
    llmq.llmq_quantize_fp8_blocks(x.to(DEV), fmt, block_rows, q, s, qt, st)
    torch.cuda.synchronize()
    return q, s, qt, st


def assert_codes(q, s, x, fmt, block_rows, what):
    codes, b = bc.quantize(x, fmt, block_rows)
    got = bc.scale_bytes(s, *x.shape)
    assert np.array_equal(got, b), "%s: scales differ at %s" % (what, np.argwhere(got != b)[:3])
    fine = ~np.isnan(codes)
    assert np.array_equal(bc.decode(q, fmt)[fine], codes[fine]), "%s: codes differ at %s" % (what, np.argwhere((bc.decode(q, fmt) != codes) & fine)[:3])


SHAPES = [(1, 1), (1, 16), (3, 7), (16, 128), (128, 1), (127, 129), (128, 128), (129, 8), (130, 131), (256, 384), (300, 200), (64, 1000), (1000, 65), (257, 513), (1, 4099)]


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_codes_and_scales_are_the_formats(rows, cols, fmt, block_rows):
    x = tensor(rows, cols, rows * 7 + cols)
    q, s, qt, st = run_quantize(x, fmt, block_rows)
    assert_codes(q, s, x, fmt, block_rows, "rows")
    assert_codes(qt, st, x.t().contiguous(), fmt, block_rows, "columns")
    if block_rows == 128:
        assert torch.equal(q.t().contiguous(), qt)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("copies", ["rows", "columns"])
@pytest.mark.parametrize("rows,cols", [(256, 256), (200, 77)])
def test_one_copy_alone_is_the_same(rows, cols, copies, block_rows):
    x = tensor(rows, cols, 5)
    both, one = run_quantize(x, 0, block_rows), run_quantize(x, 0, block_rows, copies)
    for a, b in zip(both, one):
        assert b is None or torch.equal(a, b)


@pytest.mark.parametrize("rows,cols", [(384, 512), (300, 400)])
def test_streamed_stores_and_pieces_of_a_launch(rows, cols, monkeypatch):
    x = tensor(rows, cols, 3)
    plain = run_quantize(x, 0, 1)
    monkeypatch.setenv("LLMQ_STREAM", "1")
    monkeypatch.setenv("LLMQ_MAX_WORKGROUPS", "8")
    for a, b in zip(plain, run_quantize(x, 0, 1)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_every_magnitude(fmt, block_rows):
    """Each row's largest value is another BF16 number: all exponents with mantissas around 1.75, subnormals, zeros, the largest."""
    bits = [e << 7 | m for e in range(255) for m in (0, 1, 95, 96, 97, 127)] + [0, 1, 2, 127]
    top = torch.tensor(bits, dtype=torch.int16).view(torch.bfloat16)
    g = torch.Generator().manual_seed(1)
    part = torch.rand(len(bits), 256, generator=g) * 2 - 1
    x = (top[:, None].double() * part).to(torch.bfloat16)
    x[:, 17] = top
    x[:, 200] = -top
    if block_rows == 128:
        x = torch.cat([torch.nn.functional.pad(r[None], (0, 0, 0, 127)) for r in x[::40]])
    q, s, qt, st = run_quantize(x, fmt, block_rows)
    assert_codes(q, s, x, fmt, block_rows, "rows")
    assert_codes(qt, st, x.t().contiguous(), fmt, block_rows, "columns")


def test_every_value_is_rounded_to_the_nearest():
    """All finite BF16 values of one binade and below under a scale of one: ties go to even, nothing is clipped."""
    for fmt, top in ((0, 448.0), (1, 57344.0)):
        e = int(np.frexp(top)[1]) - 1
        grid = torch.tensor([m * 2.0 ** (k - 7) for k in range(e - 30, e + 1) for m in range(128, 256)], dtype=torch.float64)
        grid = grid[grid <= top].to(torch.bfloat16)
        grid = grid[: grid.numel() // 126 * 126].view(-1, 126)
        x = torch.cat([torch.full((grid.shape[0], 1), top, dtype=torch.bfloat16), grid, torch.zeros(grid.shape[0], 1, dtype=torch.bfloat16)], 1)
        x = torch.cat([x, -x])
        q, s, qt, st = run_quantize(x, fmt, 1)
        assert (bc.scale_bytes(s, *x.shape) == 127).all()
        assert_codes(q, s, x, fmt, 1, "rows")


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_non_finite_values_spoil_their_block_alone(bad, block_rows):
    x = tensor(256, 300, 9)
    x[130, 140] = bad
    q, s, qt, st = run_quantize(x, 0, block_rows)
    b = bc.scale_bytes(s, 256, 300)
    where = b == 255
    assert where[130, 1] and where.sum() == block_rows
    assert_codes(q, s, x, 0, block_rows, "rows")
    assert_codes(qt, st, x.t().contiguous(), 0, block_rows, "columns")
    # a contraction that reads the block is NaN in its rows, and nowhere else
    other = tensor(64, 300, 10)
    p, sp, _, _ = run_quantize(other, 0, 1)
    c = torch.zeros(256, 64, device=DEV, dtype=torch.bfloat16)
    llmq.llmq_fp8_gemm_blocks(q, s, 0, p, sp, 0, c)
    nan_rows = torch.isnan(c.float()).all(1).cpu().numpy()
    assert np.array_equal(nan_rows, where.any(1)) and torch.isfinite(c.float()).cpu().numpy()[~nan_rows].all()


def operands(R, C, T, fa, fb, seed, block_b=1):
    a, b = tensor(R, T, seed, 1.0), tensor(C, T, seed + 1, 1.0)
    qa, sa, _, _ = run_quantize(a, fa, 1, "rows")
    qb, sb, _, _ = run_quantize(b, fb, block_b, "rows")
    # bytes of rows that do not exist: rubbish
    sa, sb = (bc.packed(bc.scale_bytes(s, n, T)).to(DEV) for s, n in ((sa, R), (sb, C)))
    va, vb = (bc.values(bc.decode(q, f), bc.scale_bytes(s, n, T)) for q, s, f, n in ((qa, sa, fa, R), (qb, sb, fb, C)))
    return qa, sa, qb, sb, va, vb


def assert_close(c, va, vb, T, old=None):
    """The contract's bound, 2^-7 of the products' magnitudes S (and of the old value added).  What it is made of: one rounding to BF16, 2^-8 |y| <= 2^-8 S; the
    binary32 additions from one K step to the next, one for each 128 elements, 33 2^-24 S for T up to 4224; and what the matrix cores lose inside a K step, where
    they align 128 products to the largest of them, so that a product can lose no more than itself: at most 2^-8 S is left for that, and 2^-12.3 S is the most that was
    measured (sums of BF16 results and their remainders, formats and magnitudes mixed).  That the sums are those of the contraction without block scales, bit for
    bit, is tested below."""
    y, S = va @ vb.T, np.abs(va) @ np.abs(vb).T
    if old is not None:
        o = old.cpu().to(torch.float64).numpy()
        y, S = y + o, S + np.abs(o)
    err = np.abs(c.cpu().to(torch.float64).numpy() - y)
    bound = 2.0 ** -7 * S
    assert (err <= bound).all(), "worst %g of the bound at %s" % ((err / bound).max(), np.unravel_index((err / bound).argmax(), err.shape))


GEMMS = [(1, 1, 1), (1, 8, 15), (2, 3, 16), (16, 16, 128), (17, 40, 100), (16, 300, 512), (64, 64, 640), (100, 136, 200), (128, 128, 128), (128, 256, 384),
         (256, 256, 256), (300, 520, 300), (257, 129, 1023), (512, 512, 128), (640, 768, 272), (1, 2000, 1024), (1000, 1, 130)]


@pytest.mark.parametrize("fa,fb", [(0, 0), (1, 0), (0, 1), (1, 1)])
@pytest.mark.parametrize("R,C,T", GEMMS)
def test_contraction(R, C, T, fa, fb):
    qa, sa, qb, sb, va, vb = operands(R, C, T, fa, fb, R + C + T, 128 if C % 2 else 1)
    c = torch.full((R, C), 7.0, device=DEV, dtype=torch.bfloat16)
    amax = torch.full((1,), -1.0, device=DEV)
    llmq.llmq_fp8_gemm_blocks(qa, sa, fa, qb, sb, fb, c, False, amax)
    assert_close(c, va, vb, T)
    assert amax.item() == c.abs().max().item()
    old = torch.randn(R, C, device=DEV).to(torch.bfloat16) * c.abs().max()
    c2 = old.clone()
    llmq.llmq_fp8_gemm_blocks(qa, sa, fa, qb, sb, fb, c2, True, amax)
    assert_close(c2, va, vb, T, old)
    assert amax.item() == c2.abs().max().item()
    c3 = torch.zeros_like(c)
    llmq.llmq_fp8_gemm_blocks(qa, sa, fa, qb, sb, fb, c3)
    assert torch.equal(c, c3)                              # same inputs, same bytes


TILES = ["4x4", "4x3", "4x2", "3x4", "3x3", "3x2", "2x4", "2x3", "2x2"]


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("tile", TILES + ["mini 32", "mini 64", "0x0"])
@pytest.mark.parametrize("R,C,T", [(256, 512, 128), (512, 256, 640), (512, 768, 1152), (384, 576, 256), (768, 384, 640), (300, 700, 272), (450, 333, 400), (300, 268, 1001), (129, 257, 17), (600, 520, 1664)])
def test_every_kernel(R, C, T, tile, accumulate, monkeypatch):
    if tile.startswith("mini"):
        monkeypatch.setenv("LLMQ_GEMM_MINI", tile[5:])
    else:
        monkeypatch.setenv("LLMQ_GEMM_ANY_TILE", tile)
        monkeypatch.setenv("LLMQ_GEMM_MINI", "0")
    monkeypatch.setenv("LLMQ_FEW", "0")
    for deep in ("0", "1") if tile == "2x2" else ("0",):
        monkeypatch.setenv("LLMQ_GEMM_DEEP", deep)
        qa, sa, qb, sb, va, vb = operands(R, C, T, 1, 0, R + T, 1)
        old = torch.randn(R, C, device=DEV).to(torch.bfloat16)
        c, amax = old.clone(), torch.zeros(1, device=DEV)
        llmq.llmq_fp8_gemm_blocks(qa, sa, 1, qb, sb, 0, c, accumulate, amax)
        assert_close(c, va, vb, T, old if accumulate else None)
        assert amax.item() == c.abs().max().item()


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("R,C,T,strip", [(384, 256, 128, "r128"), (256, 384, 640, "c128"), (768, 512, 384, "r256"), (512, 1152, 256, "c640"), (896, 256, 1152, "r384"), (256, 896, 2304, "c384"),
                                         (512, 768, 128, "c512"), (2048, 256, 256, "r1792")])
def test_strips(R, C, T, strip, accumulate, monkeypatch):
    """The last rows or columns in a launch of their own: the bytes of one launch, absmax too"""
    qa, sa, qb, sb, va, vb = operands(R, C, T, 1, 0, R + T, 1)
    old = torch.randn(R, C, device=DEV).to(torch.bfloat16)
    out = {}
    for how in ("0", strip):
        monkeypatch.setenv("LLMQ_BLOCKS_STRIP", how)
        c, amax = old.clone(), torch.zeros(1, device=DEV)
        llmq.llmq_fp8_gemm_blocks(qa, sa, 1, qb, sb, 0, c, accumulate, amax)
        assert_close(c, va, vb, T, old if accumulate else None)
        assert amax.item() == c.abs().max().item()
        out[how] = c
    assert torch.equal(out["0"].view(torch.int16), out[strip].view(torch.int16))


def test_a_contraction_that_is_cut_gives_the_bytes_of_one_launch(monkeypatch):
    """257 tiles of 256 x 256 and 16 K steps: a strip by the rule on sizes, no switch"""
    R, C, T = 257 * 256, 256, 2048
    qa, sa, qb, sb, _, _ = operands(R, C, T, 0, 0, 3, 1)
    outs = [torch.empty(R, C, device=DEV, dtype=torch.bfloat16) for _ in range(2)]
    llmq.llmq_fp8_gemm_blocks(qa, sa, 0, qb, sb, 0, outs[0])
    monkeypatch.setenv("LLMQ_BLOCKS_STRIP", "0")
    llmq.llmq_fp8_gemm_blocks(qa, sa, 0, qb, sb, 0, outs[1])
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))


@pytest.mark.parametrize("fa,fb", [(0, 0), (1, 0), (0, 1), (1, 1)])
@pytest.mark.parametrize("R,C,T", [(16, 40, 200), (128, 256, 384), (512, 768, 1152), (300, 700, 272), (300, 268, 1001)])
def test_scales_of_rows_alone_give_the_bytes_of_the_contraction_without_them(R, C, T, fa, fb, monkeypatch):
    """One scale for all of a row's blocks is a power of two on the result; the kernel for operands with one scale, forced to the same tile, adds in the
    same order.  Magnitudes are such that no BF16 result is subnormal."""
    tile = "2x2" if T % 16 else "4x4"
    monkeypatch.setenv("LLMQ_GEMM_ANY_TILE", tile)
    monkeypatch.setenv("LLMQ_GEMM_EDGE_TILE", tile)
    monkeypatch.setenv("LLMQ_GEMM_MINI", "0")
    g = torch.Generator().manual_seed(R)
    a, b = torch.randn(R, T, generator=g).to(bc.FLOAT8[fa]).view(torch.uint8).to(DEV), torch.randn(C, T, generator=g).to(bc.FLOAT8[fb]).view(torch.uint8).to(DEV)
    ea, eb = torch.randint(100, 150, (R, 1), generator=g), torch.randint(100, 150, (C, 1), generator=g)
    steps = bc.padded(T) // 128
    sa, sb = (bc.packed(e.expand(-1, steps).numpy()).to(DEV) for e in (ea, eb))
    one = torch.ones(1, device=DEV)
    want, got = (torch.zeros(R, C, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    llmq.llmq_fp8_gemm_tn(a, fa, b, fb, one, one, want)
    llmq.llmq_fp8_gemm_blocks(a, sa, fa, b, sb, fb, got)
    power = torch.ldexp(torch.ones(()).double(), (ea - 127) + (eb - 127).t()).to(DEV)
    assert torch.equal(got.double(), want.double() * power)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("R,C,T", [(1, 16, 16), (1, 5, 200), (3, 50, 131), (16, 64, 2048), (9, 4200, 640), (16, 100, 1999), (17, 33, 4112), (32, 4099, 512), (25, 4096, 272), (31, 1000, 777), (2, 40, 20000),
                                   (33, 40, 129), (100, 70, 1999), (130, 16, 612), (200, 333, 77), (64, 4200, 512), (257, 48, 1000), (1000, 33, 19)])
def test_few_rows(R, C, T, accumulate, monkeypatch):
    """The kernel for few rows, one and two blocks of columns to a workgroup, whole chunks and any, fewer steps than waves and many more, groups of rows."""
    monkeypatch.setenv("LLMQ_FEW", "1")
    for fa, fb in ((0, 0), (1, 0), (0, 1), (1, 1)):
        qa, sa, qb, sb, va, vb = operands(R, C, T, fa, fb, R + T, 1 if C % 2 else 128)
        old = torch.randn(R, C, device=DEV).to(torch.bfloat16)
        guard = torch.full((R * C + 64,), 3.0, device=DEV, dtype=torch.bfloat16)
        c, amax = guard[: R * C].view(R, C), torch.zeros(1, device=DEV)
        c.copy_(old)
        llmq.llmq_fp8_gemm_blocks(qa, sa, fa, qb, sb, fb, c, accumulate, amax)
        assert_close(c, va, vb, T, old if accumulate else None)
        assert amax.item() == c.abs().max().item() and (guard[R * C :] == 3.0).all()


def test_many_steps_and_tiles():
    """More tiles than compute units, and a contraction long enough for every stage to come round often."""
    R, C, T = 2304, 4352, 2176
    qa, sa, qb, sb, va, vb = operands(R, C, T, 0, 0, 3, 128)
    c = torch.zeros(R, C, device=DEV, dtype=torch.bfloat16)
    llmq.llmq_fp8_gemm_blocks(qa, sa, 0, qb, sb, 0, c)
    assert_close(c, va, vb, T)


def test_scales_at_the_ends_of_their_range():
    """Bytes 0 and 254 against each other: the products are ordinary numbers, and zero codes stay zero."""
    R, C, T = 32, 48, 256
    g = torch.Generator().manual_seed(2)
    qa, qb = (torch.randn(n, T, generator=g).to(torch.float8_e4m3fn) for n in (R, C))
    ba, bb = np.full((R, 2), 0), np.full((C, 2), 254)
    ba[:, 1], bb[:, 1] = 254, 0
    c = torch.zeros(R, C, device=DEV, dtype=torch.bfloat16)
    llmq.llmq_fp8_gemm_blocks(qa.view(torch.uint8).to(DEV), bc.packed(ba).to(DEV), 0, qb.view(torch.uint8).to(DEV), bc.packed(bb).to(DEV), 0, c)
    assert_close(c, bc.values(qa.double().numpy(), ba), bc.values(qb.double().numpy(), bb), T)


def test_a_captured_pass_follows_its_inputs():
    """Quantizers and contraction in one graph, replayed on changed inputs with eager work in between."""
    R, C, T = 300, 512, 640
    x, w = tensor(R, T, 1).to(DEV), tensor(C, T, 2).to(DEV)
    u8 = lambda n: torch.zeros(n, device=DEV, dtype=torch.uint8)  # noqa: E731
    q, s, p, sp = u8((R, T)), u8(llmq.llmq_block_scales_bytes(R, T)), u8((C, T)), u8(llmq.llmq_block_scales_bytes(C, T))
    c, amax = torch.zeros(R, C, device=DEV, dtype=torch.bfloat16), torch.zeros(1, device=DEV)

    def whole(c, amax):
        llmq.llmq_quantize_fp8_blocks(x, 0, 1, q, s)
        llmq.llmq_quantize_fp8_blocks(w, 0, 128, p, sp)
        llmq.llmq_fp8_gemm_blocks(q, s, 0, p, sp, 0, c, False, amax)

    whole(c, amax)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            whole(c, amax)
    for k in range(4):
        x.copy_(tensor(R, T, 10 + k))
        graph.replay()
        torch.cuda.synchronize()
        got, got_amax = c.clone(), amax.clone()
        c2, amax2 = torch.zeros_like(c), torch.zeros_like(amax)
        whole(c2, amax2)
        torch.cuda.synchronize()
        assert torch.equal(got, c2) and torch.equal(got_amax, amax2)


def test_bad_calls_are_refused():
    x = tensor(130, 200, 1).to(DEV)
    q, s = torch.zeros(130, 200, device=DEV, dtype=torch.uint8), torch.zeros(llmq.llmq_block_scales_bytes(130, 200), device=DEV, dtype=torch.uint8)
    with pytest.raises(llmq.LlmqError):
        llmq.llmq_quantize_fp8_blocks(x, 0, 64, q, s)                       # no such blocks
    with pytest.raises(llmq.LlmqError):
        llmq.llmq_quantize_fp8_blocks(x, 2, 1, q, s)
    with pytest.raises(llmq.LlmqError):
        llmq.llmq_quantize_fp8_blocks(x, 0, 1, None, None)
    with pytest.raises(llmq.LlmqError):
        llmq.llmq_quantize_fp8_blocks(x, 0, 1, q, None)
    with pytest.raises(ValueError):
        llmq.llmq_quantize_fp8_blocks(x, 0, 1, q, s[:-1])
    with pytest.raises(ValueError):
        llmq.llmq_quantize_fp8_blocks(x.t(), 0, 1, q, s)                    # not contiguous
    with pytest.raises(TypeError):
        llmq.llmq_quantize_fp8_blocks(x.float(), 0, 1, q, s)
    c = torch.zeros(130, 130, device=DEV, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        llmq.llmq_fp8_gemm_blocks(q, s[:-1], 0, q, s, 0, c)
    with pytest.raises(ValueError):
        llmq.llmq_fp8_gemm_blocks(q, s, 0, q, s, 0, c[:, :64].contiguous())
    with pytest.raises(ValueError):
        llmq.llmq_fp8_gemm_blocks(q.cpu(), s, 0, q, s, 0, c)
