"""The operators of a transformer block's second half around its FP8 linears, as cases to measure: what they are given, what they compute and what they cannot do without.

  norm_fwd   residual addition and RMSNorm, out as FP8 codes with a power-of-two scale for every block of 128 elements: row-wise and, for training, transposed
  norm_bwd   its gradient, with the residual stream's own gradient added: dX, and the gradient of the norm's weight
  ffn_fwd    both projections of a gated feed-forward block and the SwiGLU between them, h = silu(X Wg^T) * (X Wu^T), from operands with block scales
  ffn_bwd    the gradient through the down projection and the SwiGLU: dGU from dY, W_down and the kept GU, and h once more for the weight gradient

`own` chooses between the framework's calls and plain torch operations in binary32."""
import math

import torch

own = False
DEV = "cuda"
E4M3, E5M2 = 0, 1
FLOAT8 = {E4M3: torch.float8_e4m3fn, E5M2: torch.float8_e5m2}
EPS = 1e-6


def listed():
    return [
        # one token of each of 32 sequences in front of a projection: the row-wise codes are all that is read
        {"name": "norm 32 tokens", "op": "norm_fwd", "M": 32, "C": 3584, "fmt": E4M3, "add": True, "both": False},
        # a training step's norm: codes along the rows for the product, along the columns for the weight gradient
        {"name": "norm forward", "op": "norm_fwd", "M": 8192, "C": 3584, "fmt": E4M3, "add": True, "both": True},
        # a ragged token count
        {"name": "norm forward ragged", "op": "norm_fwd", "M": 1777, "C": 2880, "fmt": E4M3, "add": True, "both": True},
        # a micro-step of few tokens, then the backward pass of a wider layer, and of rows that are no whole vectors
        {"name": "norm backward small", "op": "norm_bwd", "M": 256, "C": 2048, "dres": True},
        {"name": "norm backward", "op": "norm_bwd", "M": 8192, "C": 5120, "dres": True},
        {"name": "norm backward ragged", "op": "norm_bwd", "M": 1777, "C": 2730, "dres": True},
        # sixteen tokens through the gate and up projections: the weights are all there is to read
        {"name": "ffn 16 tokens", "op": "ffn_fwd", "M": 16, "I": 18944, "T": 3584, "fmt_a": E4M3, "keep": False},
        # the forward product in training, which keeps the gate and up branches
        {"name": "ffn forward", "op": "ffn_fwd", "M": 8192, "I": 18944, "T": 3584, "fmt_a": E4M3, "keep": True},
        # a prompt of odd length through a small layer
        {"name": "ffn forward ragged", "op": "ffn_fwd", "M": 1777, "I": 2720, "T": 1000, "fmt_a": E4M3, "keep": False},
        # its gradient; output gradients in the format with the wider range
        {"name": "ffn backward", "op": "ffn_bwd", "M": 8192, "I": 18944, "T": 3584, "fmt_a": E5M2, "h": True},
        {"name": "ffn backward ragged", "op": "ffn_bwd", "M": 1777, "I": 2720, "T": 1000, "fmt_a": E5M2, "h": False},
        # the gradient of a short sequence
        {"name": "ffn backward 512 tokens", "op": "ffn_bwd", "M": 512, "I": 8192, "T": 2048, "fmt_a": E4M3, "h": True},
    ]


def _spread(rng, low, high):
    """A whole number between low and high, spread over the logarithm."""
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "ffn_fwd", "ffn_fwd", "ffn_bwd", "ffn_bwd"])
    if op in ("norm_fwd", "norm_bwd"):
        M, C = _spread(rng, 1, 8192), _spread(rng, 64, 5120)
        if rng.random() < 0.5:
            C = 64 * -(-C // 64)
        if op == "norm_fwd":
            return {"op": op, "M": M, "C": C, "fmt": rng.choice([E4M3, E4M3, E5M2]), "add": rng.random() < 0.8, "both": rng.random() < 0.6}
        return {"op": op, "M": M, "C": C, "dres": rng.random() < 0.8}
    M, I, T = _spread(rng, 1, 8192), _spread(rng, 64, 18944), _spread(rng, 64, 3584)
    if rng.random() < 0.7:
        I, T = (64 * -(-v // 64) for v in (I, T))
    fmt_a = rng.choice([E4M3, E4M3, E5M2])
    return {"op": op, "M": M, "I": I, "T": T, "fmt_a": fmt_a} | ({"keep": rng.random() < 0.5} if op == "ffn_fwd" else {"h": rng.random() < 0.5})


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 17)
    return g


def _randn(g, *shape, std=1.0):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32) * std


def _activations(g, rows, cols):
    """Gaussian values whose rows and columns differ in size, some columns far larger than the others."""
    x = _randn(g, rows, cols)
    x *= torch.exp(_randn(g, rows, 1, std=0.5))
    x *= torch.where(torch.rand(1, cols, generator=g, device=DEV) < 0.005, 30.0, 1.0)
    return x.to(torch.bfloat16)


# ---- blocks of 128 in 8 bits

def _pad128(n):
    return -(-n // 128) * 128


def _power(b):
    """2^(b - 127) of whole numbers b."""
    return torch.ldexp(torch.ones_like(b, dtype=torch.float64), b - 127).float()


def _exponents(amax, fmt):
    """The code b of each block's scale: 2^(b - 127) is the smallest power of two that brings the absmax to at most the format's largest value, 1.75 2^8 or 1.75 2^15."""
    mantissa, e = torch.frexp(amax)
    b = e - 1 - (8 if fmt == E4M3 else 15) + (mantissa > 0.875).int() + 127
    return torch.where(amax == 0, torch.full_like(b, 127), b.clamp(min=0))


def _interleave(b):
    """Codes [rows padded, K steps] in the order in which they are kept: K step by K step, 128 rows at a time, row r at 8 (r % 16) + r / 16."""
    steps = b.shape[1]
    return b.reshape(-1, 8, 16, steps).permute(3, 0, 2, 1).reshape(steps, -1).to(torch.uint8)


def _rows_of(s, rows):
    """The scales [rows, K steps] that such codes stand for."""
    steps = s.shape[0]
    return _power(s.reshape(steps, -1, 16, 8).permute(1, 3, 2, 0).reshape(-1, steps)[:rows].int())


def _plain_quantize(x, fmt, block_rows):
    """Codes and scales of x [rows, cols] in blocks of block_rows x 128 along the columns."""
    rows, cols = x.shape
    padded = torch.zeros(_pad128(rows), _pad128(cols), device=x.device, dtype=torch.float32)
    padded[:rows, :cols] = x
    blocks = padded.view(padded.shape[0] // block_rows, block_rows, -1, 128)
    b = _exponents(blocks.abs().amax(dim=(1, 3)), fmt)
    codes = (blocks * _power(254 - b)[:, None, :, None]).reshape(padded.shape)[:rows, :cols].to(FLOAT8[fmt])
    return codes.contiguous(), _interleave(b.repeat_interleave(block_rows, 0))


def _dequantized(q, s, fmt):
    scale = _rows_of(s, q.shape[0]).repeat_interleave(128, 1)[:, : q.shape[1]]
    return q.view(FLOAT8[fmt]).float() * scale


def _scales(s):
    """Scale bytes as the powers of two they stand for."""
    return s.view(torch.float8_e8m0fnu)


# ---- the plain forms

def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _plain_norm_fwd(st):
    c = st["case"]
    res = st["res"].float()
    if c["add"]:
        res = (res + st["x"].float()).to(torch.bfloat16)
    r = res.float()
    rstd = 1.0 / torch.sqrt((r * r).mean(-1) + EPS)
    y = (r * rstd[:, None] * st["w"].float()).to(torch.bfloat16)
    q, s = _plain_quantize(y, c["fmt"], 1)
    out = [rstd, q, _scales(s)] + ([res] if c["add"] else [])
    if c["both"]:
        q_t, s_t = _plain_quantize(y.t(), c["fmt"], 1)
        out += [q_t, _scales(s_t)]
    return out


def _plain_norm_bwd(st):
    dy, r = st["dy"].float(), st["rstd"][:, None]
    n = st["res"].float() * r
    dw = (dy * n).sum(0)
    g = dy * st["w"].float()
    dx = r * (g - n * (g * n).mean(-1, keepdim=True))
    if st["case"]["dres"]:
        dx = dx + st["dres"].float()
    return [dx.to(torch.bfloat16), dw]


def _plain_ffn_fwd(st):
    c = st["case"]
    gu = torch.matmul(_dequantized(st["a"], st["s_a"], c["fmt_a"]), _dequantized(st["b"], st["s_b"], E4M3).t())
    gate, up = gu[:, : c["I"]], gu[:, c["I"] :]
    h = (gate * _sigmoid(gate) * up).to(torch.bfloat16)
    return [h] + ([gu.to(torch.bfloat16)] if c["keep"] else [])


def _plain_ffn_bwd(st):
    c = st["case"]
    dh = torch.matmul(_dequantized(st["a"], st["s_a"], c["fmt_a"]), _dequantized(st["b"], st["s_b"], E4M3).t())
    gate, up = st["gu"][:, : c["I"]].float(), st["gu"][:, c["I"] :].float()
    sg = _sigmoid(gate)
    dgu = torch.cat((dh * up * sg * (1 + gate * (1 - sg)), dh * gate * sg), 1).to(torch.bfloat16)
    return [dgu] + ([(gate * sg * up).to(torch.bfloat16)] if c["h"] else [])


# ---- what the tools call

def prepare(case, seed):
    g, op = _generator(seed), case["op"]
    st = {"case": case}
    bf16 = {"device": DEV, "dtype": torch.bfloat16}
    u8 = {"device": DEV, "dtype": torch.uint8}
    if op == "norm_fwd":
        M, C = case["M"], case["C"]
        st["res"] = _activations(g, M, C)
        st["x"] = _randn(g, M, C, std=0.3).to(torch.bfloat16) if case["add"] else None
        st["w"] = (1 + _randn(g, C, std=0.1)).to(torch.bfloat16)
        st["res_out"] = torch.empty(M, C, **bf16) if case["add"] else None
        st["rstd"] = torch.empty(M, device=DEV)
        st["q"], st["s"] = torch.empty(M, C, **u8), torch.empty(_pad128(C) // 128, _pad128(M), **u8)
        st["q_t"], st["s_t"] = (torch.empty(C, M, **u8), torch.empty(_pad128(M) // 128, _pad128(C), **u8)) if case["both"] else (None, None)
    elif op == "norm_bwd":
        M, C = case["M"], case["C"]
        st["res"] = _activations(g, M, C)
        st["w"] = (1 + _randn(g, C, std=0.1)).to(torch.bfloat16)
        r = st["res"].float()
        st["rstd"] = 1.0 / torch.sqrt((r * r).mean(-1) + EPS)
        st["dy"] = (_randn(g, M, C, std=1e-3) * torch.exp(_randn(g, M, 1, std=0.5))).to(torch.bfloat16)
        st["dres"] = _randn(g, M, C, std=1e-3).to(torch.bfloat16) if case["dres"] else None
        st["dx"], st["dw"] = torch.empty(M, C, **bf16), torch.empty(C, device=DEV)
        if own:
            from paper_2512_15306_amd import llmq
            st["ws"] = torch.empty(llmq.llmq_rmsnorm_bwd_workspace_bytes(M, C), **u8)
    else:
        M, I, T = case["M"], case["I"], case["T"]
        if op == "ffn_fwd":
            a, st["s_a"] = _plain_quantize(_activations(g, M, T), case["fmt_a"], 1)
            # gate and up rows of one weight; sums of about one
            b, st["s_b"] = _plain_quantize(_randn(g, 2 * I, T, std=0.7 / math.sqrt(T)).to(torch.bfloat16), E4M3, 128)
            st["h"] = torch.empty(M, I, **bf16)
            st["gu"] = torch.empty(M, 2 * I, **bf16) if case["keep"] else None
        else:
            dy = _randn(g, M, T, std=1e-3) * torch.exp(_randn(g, M, 1, std=0.5))
            a, st["s_a"] = _plain_quantize(dy.to(torch.bfloat16), case["fmt_a"], 1)
            # the transposed copy of the down projection's weight
            b, st["s_b"] = _plain_quantize(_randn(g, I, T, std=1 / math.sqrt(I)).to(torch.bfloat16), E4M3, 128)
            st["gu"] = (_randn(g, M, 2 * I) * torch.exp(_randn(g, M, 1, std=0.5))).to(torch.bfloat16)
            st["dgu"] = torch.empty(M, 2 * I, **bf16)
            st["h"] = torch.empty(M, I, **bf16) if case["h"] else None
        st["a"], st["b"] = a.view(torch.uint8), b.view(torch.uint8)
    return st


def run(st):
    case = st["case"]
    op = case["op"]
    if own:
        from paper_2512_15306_amd import llmq
        if op == "norm_fwd":
            llmq.llmq_rmsnorm_fwd_fp8_blocks(st["res"], st["x"], st["w"], EPS, st["res_out"], st["rstd"], case["fmt"], st["q"], st["s"], st["q_t"], st["s_t"])
            codes = FLOAT8[case["fmt"]]
            return [st["rstd"], st["q"].view(codes), _scales(st["s"])] + ([st["res_out"]] if case["add"] else []) + ([st["q_t"].view(codes), _scales(st["s_t"])] if case["both"] else [])
        if op == "norm_bwd":
            llmq.llmq_rmsnorm_bwd(st["dy"], st["dres"], st["res"], st["w"], st["rstd"], st["dx"], st["dw"], False, E5M2, None, None, st["ws"])
            return [st["dx"], st["dw"]]
        if op == "ffn_fwd":
            llmq.llmq_fp8_gemm_blocks_swiglu_fwd(st["a"], st["s_a"], case["fmt_a"], st["b"], st["s_b"], E4M3, st["h"], st["gu"])
            return [st["h"]] + ([st["gu"]] if case["keep"] else [])
        llmq.llmq_fp8_gemm_blocks_swiglu_bwd(st["a"], st["s_a"], case["fmt_a"], st["b"], st["s_b"], E4M3, st["gu"], st["dgu"], st["h"])
        return [st["dgu"]] + ([st["h"]] if case["h"] else [])
    return {"norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd, "ffn_fwd": _plain_ffn_fwd, "ffn_bwd": _plain_ffn_bwd}[op](st)


def work(case):
    op, M = case["op"], case["M"]
    steps = lambda n: -(-n // 128)  # noqa: E731
    if op == "norm_fwd":
        n = M * case["C"]
        codes = n + M * steps(case["C"]) + (n + case["C"] * steps(M) if case["both"] else 0)
        return {"bytes": (6 if case["add"] else 2) * n + codes + 4 * M + 2 * case["C"], "flops": 10 * n}
    if op == "norm_bwd":
        n = M * case["C"]
        return {"bytes": (8 if case["dres"] else 6) * n + 4 * M + 6 * case["C"], "flops": 12 * n}
    I, T = case["I"], case["T"]
    if op == "ffn_fwd":
        return {"bytes": (M + 2 * I) * (T + steps(T)) + (6 if case["keep"] else 2) * M * I, "flops": 4 * M * I * T}
    return {"bytes": (M + I) * (T + steps(T)) + (10 if case["h"] else 8) * M * I, "flops": 2 * M * I * T}


# ---- the same in binary64, from the definitions

def _two_to(e):
    return torch.pow(2.0, e).float().double()            # exact, which the power of the device need not be


def _floor_log2(x):
    return torch.frexp(x.clamp(min=2.0**-300))[1].double() - 1


def _ceil_log2(x):
    mantissa, e = torch.frexp(x.clamp(min=2.0**-300))
    return e.double() - (mantissa == 0.5).double()


def _grid(y, mantissa_bits, least):
    """y at the nearest value with so many mantissa bits, ties to even; below 2^least the spacing stays."""
    step = _two_to(_floor_log2(y.abs()).clamp(min=least) - mantissa_bits)
    return torch.round(y / step) * step


def _exact_codes(x, fmt):
    largest, bits, least = (448.0, 3, -6) if fmt == E4M3 else (57344.0, 2, -14)
    rows, cols = x.shape
    y = torch.zeros(rows, _pad128(cols), device=x.device, dtype=torch.float64)
    y[:, :cols] = x
    y = y.view(rows, -1, 128)
    d = _two_to(_ceil_log2(y.abs().amax(2, keepdim=True) / largest).clamp(min=-127))
    return _grid(y / d, bits, least).reshape(rows, -1)[:, :cols]


def _exact_values(q, s, fmt):
    r = torch.arange(q.shape[0], device=q.device)
    place = (r // 128) * 128 + (r % 16) * 8 + (r % 128) // 16
    return q.view(FLOAT8[fmt]).double() * _two_to(s.double() - 127)[:, place].t().repeat_interleave(128, 1)[:, : q.shape[1]]


def exact(case, seed):
    op, st = case["op"], prepare(case, seed)
    if op == "norm_fwd":
        res = st["res"].double()
        if case["add"]:
            res = _grid(res + st["x"].double(), 7, -126)
        inverse = (res.square().mean(-1) + EPS).rsqrt()
        y = _grid(res * inverse[:, None] * st["w"].double(), 7, -126)
        out = [inverse, _exact_codes(y, case["fmt"]), None] + ([res] if case["add"] else [])
        return out + ([_exact_codes(y.t(), case["fmt"]), None] if case["both"] else [])
    if op == "norm_bwd":
        # through y = x r w with r = (mean x^2 + eps)^(-1/2):  dx = r w dy - x r^3 / C sum(w dy x)
        x, r, wdy = st["res"].double(), st["rstd"].double(), st["dy"].double() * st["w"].double()
        dx = wdy * r[:, None] - x * (r**3 * (wdy * x).sum(-1) / case["C"])[:, None]
        if case["dres"]:
            dx += st["dres"].double()
        return [dx, torch.einsum("mc,mc,m->c", st["dy"].double(), x, r)]
    product = _exact_values(st["a"], st["s_a"], case["fmt_a"]) @ _exact_values(st["b"], st["s_b"], E4M3).t()
    gate, up = (product if op == "ffn_fwd" else st["gu"].double()).chunk(2, 1)
    e = torch.exp(-gate)
    h = gate * up / (1 + e)
    if op == "ffn_fwd":
        return [h] + ([product] if case["keep"] else [])
    return [torch.cat((product * up * (1 + e + gate * e) / (1 + e) ** 2, product * gate / (1 + e)), 1)] + ([h] if case["h"] else [])
