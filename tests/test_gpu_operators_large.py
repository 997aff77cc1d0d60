"""Tensors beyond 2^31 and 2^32 elements: what lies at their ends comes out as it does by itself (the small calls are checked against binary64 in the other files)."""
import pytest
import torch

from paper_2512_15306_amd import llmq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(autouse=True)
def memory():
    if torch.cuda.mem_get_info()[0] < 64 << 30:
        pytest.skip("64 GB of device memory are not free")
    yield
    torch.cuda.empty_cache()


def u8(*n):
    return torch.zeros(n, device=DEV, dtype=torch.uint8)


def scale_rows(s, rows, cols, first, count):
    """The bytes of whole groups of 128 rows"""
    return s.view((cols + 127) // 128, (rows + 127) // 128 * 128)[:, first : first + (count + 127) // 128 * 128]


def random(*n, seed=1):
    return torch.randn(*n, device=DEV, generator=torch.Generator(DEV).manual_seed(seed)).to(torch.bfloat16)


@pytest.mark.parametrize("rows,cols", [(65792, 65664), (65793, 65665)])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantizer(rows, cols, block_rows):
    """4.3 billion elements, whole tiles and ragged ones: the last rows, which lie beyond 2^32 elements"""
    n = 256 + rows % 128
    x = torch.zeros(rows, cols, device=DEV, dtype=torch.bfloat16)
    x[-n:] = random(n, cols)
    q, s, qt, st = u8(rows, cols), u8(llmq.llmq_block_scales_bytes(rows, cols)), u8(cols, rows), u8(llmq.llmq_block_scales_bytes(cols, rows))
    llmq.llmq_quantize_fp8_blocks(x, llmq.E4M3, block_rows, q, s, qt, st)
    part = x[-n:].clone()
    p, ps, pt, pst = u8(n, cols), u8(llmq.llmq_block_scales_bytes(n, cols)), u8(cols, n), u8(llmq.llmq_block_scales_bytes(cols, n))
    llmq.llmq_quantize_fp8_blocks(part, llmq.E4M3, block_rows, p, ps, pt, pst)
    assert torch.equal(q[-n:], p) and torch.equal(qt[:, -n:], pt) and p.any()
    assert torch.equal(scale_rows(s, rows, cols, rows - n, n), scale_rows(ps, n, cols, 0, n))
    assert torch.equal(st.view(-1, (cols + 127) // 128 * 128)[-((n + 127) // 128) :], pst.view(-1, (cols + 127) // 128 * 128))
    assert not q[:-n].any() and (scale_rows(s, rows, cols, 0, rows - n) == 127).all()


@pytest.mark.parametrize("R,C,T,n", [(1100800, 256, 4096, 512), (1100001, 130, 4096, 609), (530000, 136, 8200, 208)])
def test_contraction(R, C, T, n):
    """An operand beyond 2^32 bytes: whole tiles, ragged ones, rows that are no whole chunks.  Codes and scales of the last rows alone are not zeros."""
    g = torch.Generator(DEV).manual_seed(2)
    first = (R - n) // 128 * 128
    n = R - first
    A, sA = u8(R, T), torch.full((llmq.llmq_block_scales_bytes(R, T),), 127, device=DEV, dtype=torch.uint8)
    A[first:] = torch.randn(n, T, device=DEV, generator=g).to(torch.float8_e4m3fn).view(torch.uint8)
    scales = torch.randint(120, 130, ((T + 127) // 128, (n + 127) // 128 * 128), device=DEV, generator=g).to(torch.uint8)
    scale_rows(sA, R, T, first, n).copy_(scales)
    B = torch.randn(C, T, device=DEV, generator=g).to(torch.float8_e5m2).view(torch.uint8)
    sB = torch.randint(120, 130, (llmq.llmq_block_scales_bytes(C, T),), device=DEV, generator=g).to(torch.uint8)
    c, part = torch.full((R, C), 7.0, device=DEV, dtype=torch.bfloat16), torch.zeros(n, C, device=DEV, dtype=torch.bfloat16)
    llmq.llmq_fp8_gemm_blocks(A, sA, llmq.E4M3, B, sB, llmq.E5M2, c)
    llmq.llmq_fp8_gemm_blocks(A[first:].clone(), scales.reshape(-1).contiguous(), llmq.E4M3, B, sB, llmq.E5M2, part)
    assert not c[:first].any() and part.any(1).all()
    # kernels may add in another order: half a step of BF16 each, and a step of 2^-12 of the sum of the products' magnitudes (bounded by the rows' norms) that the instruction loses
    a = A[first:].view(torch.float8_e4m3fn).float() * torch.exp2(scales.view(-1, (n + 127) // 128, 16, 8).transpose(2, 3).reshape(-1, (n + 127) // 128 * 128)[:, :n].float() - 127).t().repeat_interleave(128, 1)[:, :T]
    b = B.view(torch.float8_e5m2).float() * torch.exp2(sB.view(-1, (C + 127) // 128, 16, 8).transpose(2, 3).reshape(-1, (C + 127) // 128 * 128)[:, :C].float() - 127).t().repeat_interleave(128, 1)[:, :T]
    exact, size = a.double() @ b.double().t(), a.double().abs() @ b.double().abs().t()
    for got in (part, c[first:]):
        assert ((got.double() - exact).abs() <= 2.0 ** -7 * size).all()


@pytest.mark.parametrize("D,rot", [(128, 128), (33, 32)])
def test_query_and_key_heads(D, rot):
    """Rows 4 million elements apart, the last ones beyond 2^32 elements"""
    M, Hq, Hkv, stride = 1100, 4, 2, 4_000_000
    width = (Hq + 2 * Hkv) * D
    far = torch.empty(M * stride, device=DEV, dtype=torch.bfloat16).view(M, stride)
    near, dq, dk, dv = random(M, width), random(M, Hq * D, seed=2), random(M, Hkv * D, seed=3), random(M, Hkv * D, seed=4)
    wq, wk = random(D, seed=5), random(D, seed=6)
    positions, freq = torch.arange(M, device=DEV), 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    ws = u8(llmq.llmq_qk_norm_rope_workspace_bytes(M, Hq, Hkv, D))
    place = iter(range(0, stride, 8 * 1024))

    def apart(t):
        at = next(place)
        view = far[:, at : at + t.shape[1]]
        view.copy_(t)
        return view

    def run(put):
        x, q, k, rstd = put(near), put(torch.zeros_like(dq)), put(torch.zeros_like(dk)), torch.zeros(M, Hq + Hkv, device=DEV)
        llmq.llmq_qk_norm_rope_fwd(x, Hq, Hkv, D, wq, wk, 1e-6, positions, freq, False, q, k, rstd)
        dx, dwq, dwk, a, s = put(torch.zeros_like(near)), torch.zeros(D, device=DEV), torch.zeros(D, device=DEV), torch.zeros(1, device=DEV), torch.zeros(1, device=DEV)
        llmq.llmq_qk_norm_rope_bwd(put(dq), put(dk), put(dv), x, Hq, Hkv, D, wq, wk, rstd, positions, freq, False, dx, dwq, dwk, False, llmq.E5M2, a, s, ws)
        return [t.clone() for t in (q, k, rstd, dx, dwq, dwk, a, s)]

    for one, other in zip(run(lambda t: t), run(apart)):
        assert torch.equal(one, other) and one.any()


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw(bits):
    """A tensor of more than 2^32 elements: its last ones as a tensor of their own that takes the same random numbers"""
    n, last = (1 << 32) + 12345, 128 * 100 + 57
    first = n - last
    scales, state = (n + 127) // 128, torch.uint8 if bits == 8 else torch.float32
    assert first % 128 == 0
    w, g, m, v = torch.zeros(n, device=DEV, dtype=torch.bfloat16), torch.zeros(n, device=DEV, dtype=torch.bfloat16), torch.zeros(n, device=DEV, dtype=state), torch.zeros(n, device=DEV, dtype=state)
    ms, vs = (torch.full((scales,), 127, device=DEV, dtype=torch.uint8) for _ in range(2)) if bits == 8 else (None, None)
    w[first:], g[first:] = random(last, seed=1), random(last, seed=2)
    amax = torch.zeros(2, device=DEV)
    own = [t[first:].clone() for t in (w, g, m, v)]
    own_scales = [None if t is None else t[first // 128 :].clone() for t in (ms, vs)]
    whole = llmq.AdamWTensor(w, None, g, m, v, ms, vs, 0, True, True, amax[:1])
    part = llmq.AdamWTensor(own[0], None, own[1], own[2], own[3], own_scales[0], own_scales[1], first, True, True, amax[1:])
    hyper = llmq.llmq_adamw_hyper(1, 1e-2, 0.9, 0.95, 1e-8, 0.1, 7)
    for t in (whole, part):
        llmq.llmq_adamw_step(llmq.llmq_adamw_plan([t]), hyper)
    assert torch.equal(w[first:], own[0]) and torch.equal(m[first:], own[2]) and torch.equal(v[first:], own[3]) and own[2].any()
    assert amax[0] == amax[1] > 0 and not w[:first].any()
    if bits == 8:
        assert torch.equal(ms[first // 128 :], own_scales[0]) and torch.equal(vs[first // 128 :], own_scales[1])
