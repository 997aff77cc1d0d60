"""The operators of a training step around the FP8 linears, as cases to measure: what they are given, what they compute and what they cannot do without.

  quantize   BF16 -> FP8 codes with a power-of-two scale for every block of 128 elements, row-wise and transposed copy in one call
  gemm       the contraction of two such operands, c[r, n] = sum_t A[r, t] B[n, t], BF16 out
  qk_fwd     queries and keys of a QKV projection: RMSNorm of every head and the rotation by position, in one pass
  qk_bwd     its gradient: dQKV, and the gradients of the two norm weights
  adamw      one AdamW step over many tensors, moments in binary32 or in 8 bits

`own` chooses between the framework's calls and plain torch operations in binary32 (angles of positions in binary64)."""
import math

import torch

own = False
DEV = "cuda"
E4M3, E5M2 = 0, 1
FLOAT8 = {E4M3: torch.float8_e4m3fn, E5M2: torch.float8_e5m2}
EPS = 1e-6


def listed():
    return [
        # activations of an ordinary layer on their way into the forward product (row-wise copy) and the weight gradient (transposed copy)
        {"name": "quantize 8192x3584", "op": "quantize", "rows": 8192, "cols": 3584, "fmt": E4M3, "block_rows": 1},
        # output gradients of a ragged token count, in the format with the wider range
        {"name": "quantize ragged e5m2", "op": "quantize", "rows": 1777, "cols": 4608, "fmt": E5M2, "block_rows": 1},
        # sixteen tokens through a QKV projection: the weight is all there is to read
        {"name": "gemm 16 tokens", "op": "gemm", "R": 16, "C": 4608, "T": 3584, "fmt_a": E4M3, "fmt_b": E4M3, "b_rows": 128, "accumulate": False},
        # its forward product in training
        {"name": "gemm forward", "op": "gemm", "R": 8192, "C": 4608, "T": 3584, "fmt_a": E4M3, "fmt_b": E4M3, "b_rows": 128, "accumulate": False},
        # the weight gradient of a down projection, added to what earlier micro-steps left
        {"name": "gemm weight gradient", "op": "gemm", "R": 3584, "C": 18944, "T": 8192, "fmt_a": E5M2, "fmt_b": E4M3, "b_rows": 1, "accumulate": True},
        # an input gradient of odd sizes
        {"name": "gemm ragged", "op": "gemm", "R": 1777, "C": 2880, "T": 1000, "fmt_a": E5M2, "fmt_b": E4M3, "b_rows": 128, "accumulate": False},
        # one token of each of 32 sequences, far into their contexts
        {"name": "qk 32 tokens", "op": "qk_fwd", "M": 32, "Hq": 28, "Hkv": 4, "D": 128, "rot": 128, "interleaved": False, "norm": True, "far": 100000},
        {"name": "qk forward", "op": "qk_fwd", "M": 8192, "Hq": 28, "Hkv": 4, "D": 128, "rot": 128, "interleaved": False, "norm": True, "far": 8192},
        # the backward pass of a wider layer, and of small heads of which a part is rotated, neighbours paired
        {"name": "qk backward", "op": "qk_bwd", "M": 8192, "Hq": 40, "Hkv": 8, "D": 128, "rot": 128, "interleaved": False, "norm": True, "far": 8192},
        {"name": "qk backward ragged", "op": "qk_bwd", "M": 1777, "Hq": 9, "Hkv": 3, "D": 80, "rot": 40, "interleaved": True, "norm": True, "far": 4096},
        # the weights of one transformer block, moments in 8 bits, BF16 weights with a binary32 master copy
        {"name": "adamw block 8 bit", "op": "adamw", "hidden": 3584, "qkv": 4608, "inter": 18944, "layers": 1, "bits": 8, "master": True},
        # many small tensors of odd sizes, moments in binary32
        {"name": "adamw many small", "op": "adamw", "hidden": 321, "qkv": 500, "inter": 811, "layers": 12, "bits": 32, "master": True},
    ]


def _spread(rng, low, high):
    """A whole number between low and high, spread over the logarithm."""
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))


def draw(rng):
    op = rng.choice(["quantize", "gemm", "gemm", "qk_fwd", "qk_bwd", "adamw"])
    if op == "quantize":
        return {"op": op, "rows": _spread(rng, 1, 8192), "cols": _spread(rng, 16, 3584), "fmt": rng.choice([E4M3, E5M2]), "block_rows": rng.choice([1, 1, 128])}
    if op == "gemm":
        R, C, T = _spread(rng, 1, 8192), _spread(rng, 16, 8192), _spread(rng, 16, 8192)
        if rng.random() < 0.5:
            R, C, T = (16 * -(-v // 16) for v in (R, C, T))
        return {"op": op, "R": R, "C": C, "T": T, "fmt_a": rng.choice([E4M3, E4M3, E5M2]), "fmt_b": E4M3, "b_rows": rng.choice([1, 128]), "accumulate": rng.random() < 0.3}
    if op in ("qk_fwd", "qk_bwd"):
        D = rng.choice([64, 80, 96, 128, 128, 128, 192, 256])
        Hkv = rng.choice([1, 2, 4, 8])
        Hq = Hkv * rng.choice([1, 2, 4, 5, 7])
        most = 8192 if Hq * D <= 5120 else 4096
        return {"op": op, "M": _spread(rng, 1, most), "Hq": Hq, "Hkv": Hkv, "D": D, "rot": rng.choice([D, D, D // 2]), "interleaved": rng.random() < 0.3,
                "norm": rng.random() < 0.8, "far": _spread(rng, 100, 1 << 20)}
    hidden = _spread(rng, 16, 1024)
    return {"op": op, "hidden": hidden, "qkv": _spread(rng, hidden, 3 * hidden), "inter": _spread(rng, hidden, 4 * hidden), "layers": rng.randint(1, 6), "bits": rng.choice([8, 32]),
            "master": rng.random() < 0.5}


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 17)
    return g


def _randn(g, *shape, std=1.0):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32) * std


def _activations(g, rows, cols):
    """Gaussian values whose rows and columns differ in size, some columns a hundred times the others."""
    x = _randn(g, rows, cols)
    x *= torch.exp(_randn(g, rows, 1, std=0.7))
    x *= torch.where(torch.rand(1, cols, generator=g, device=DEV) < 0.005, 100.0, 1.0)
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


def _interleave(b, rows):
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
    return codes.contiguous(), _interleave(b.repeat_interleave(block_rows, 0), rows)


def _dequantized(q, s, fmt):
    scale = _rows_of(s, q.shape[0]).repeat_interleave(128, 1)[:, : q.shape[1]]
    return q.view(FLOAT8[fmt]).float() * scale


# ---- queries and keys

def _angles(st):
    a = st["positions"].double()[:, None] * st["inv_freq"][None, :]
    return torch.cos(a).float()[:, None, :], torch.sin(a).float()[:, None, :]


def _rotated(x, cos, sin, case):
    """x [M, H, D] with the first `rot` values of every head turned."""
    r = case["rot"]
    if case["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., : r // 2], x[..., r // 2 : r]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, x[..., r:]), -1)


def _heads(x, first, count, D):
    return x[:, first * D : (first + count) * D].float().view(x.shape[0], count, D)


def _plain_qk_fwd(st):
    c = st["case"]
    cos, sin = _angles(st)
    out, stats = [], []
    for first, count, w in ((0, c["Hq"], st["wq"]), (c["Hq"], c["Hkv"], st["wk"])):
        x = _heads(st["qkv"], first, count, c["D"])
        if c["norm"]:
            rstd = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
            stats.append(rstd[..., 0])
            x = x * rstd * w.float()
        out.append(_rotated(x, cos, sin, c).to(torch.bfloat16).flatten(1))
    return out + ([torch.cat(stats, 1)] if c["norm"] else [])


def _plain_qk_bwd(st):
    c = st["case"]
    cos, sin = _angles(st)
    D, both = c["D"], c["Hq"] + c["Hkv"]
    parts, dws = [], []
    for first, count, w, dy in ((0, c["Hq"], st["wq"], st["dq"]), (c["Hq"], c["Hkv"], st["wk"], st["dk"])):
        g = _rotated(dy.float().view(-1, count, D), cos, -sin, c)
        if c["norm"]:
            rstd = st["rstd"][:, first : first + count, None]
            n = _heads(st["qkv"], first, count, D) * rstd
            dws.append((g * n).flatten(0, 1).sum(0))
            g = g * w.float()
            g = rstd * (g - n * (g * n).mean(-1, keepdim=True))
        parts.append(g.to(torch.bfloat16).flatten(1))
    dqkv = torch.cat(parts + [st["dv"]], 1)
    return [dqkv] + dws + [dqkv.abs().amax().float().view(1)]


# ---- AdamW

LR, BETA1, BETA2, DELTA, DECAY, STEP, SEED = 3e-4, 0.9, 0.95, 1e-8, 0.1, 7, 1234


def _sizes(case):
    """Sizes of the tensors of `layers` blocks: the matrices, which decay, then the norm weights, which do not."""
    h, n = case["hidden"], case["layers"]
    return n * [case["qkv"] * h, h * h, 2 * case["inter"] * h, h * case["inter"]], n * [h, h, 128, 128]


def _mixed(counter, key):
    """32 bits for every counter, as whole numbers in 64."""
    x = (counter * 0x9E3779B1 + key) & 0xFFFFFFFF
    x = ((x ^ (x >> 16)) * 0x6A09E667) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _key(step):
    """The key of a step: the mixed bits of the step number under the seed's."""
    return int(_mixed(torch.tensor(step), int(_mixed(torch.tensor(SEED), 0))))


def _eight_bits(a, rnd):
    """E4M3 codes of magnitudes a <= 448: to one of the two neighbours by 16 random bits, below 2^-6 to the nearest."""
    normal = ((a.view(torch.int32) + (rnd << 4).int()) >> 20) - 960
    return torch.where(a >= 2.0**-6, normal, torch.round(a * 512).int())


def _plain_adamw(st):
    c, n = st["case"], st["w"].numel()
    f = torch.tensor([BETA1, BETA2, 1 - BETA1, 1 - BETA2, LR, LR * DECAY, LR / (1 - BETA1**STEP), 1 / math.sqrt(1 - BETA2**STEP), DELTA], dtype=torch.float64).float().tolist()
    g, w = st["g"].float(), (st["master"] if c["master"] else st["w"]).float()
    if c["bits"] == 8:
        m = st["m"].view(torch.float8_e4m3fn).float() * _power(st["m_scale"].int()).repeat_interleave(128)
        r = st["v"].view(torch.float8_e4m3fn).float() * _power(st["v_scale"].int()).repeat_interleave(128)
        v = r * r
    else:
        m, v = st["m"], st["v"]
    m = m * f[0] + g * f[2]
    v = v * f[1] + (g * g) * f[3]
    root = torch.sqrt(v)
    decayed = w - w * torch.where(torch.arange(n, device=w.device) < st["split"], f[5], 0.0)
    w = decayed - (m / (root * f[7] + f[8])) * f[6]
    counter = torch.arange(n, device=w.device)
    if c["bits"] == 8:
        rnd = _mixed(counter, st["key"])
        for name, x, bits in (("m", m, rnd & 0xFFFF), ("v", root, rnd >> 16)):
            b = _exponents(x.abs().view(-1, 128).amax(1), E4M3)
            a = x.abs() * _power(254 - b).repeat_interleave(128)
            code = _eight_bits(a, bits)
            code = torch.where((code == 0) & (x > 0), 1, code) if name == "v" else torch.where(x < 0, code + 128, code)
            st[name].copy_(code.to(torch.uint8))
            st[name + "_scale"].copy_(b.to(torch.uint8))
    else:
        st["m"].copy_(m)
        st["v"].copy_(v)
    if c["master"]:
        st["master"].copy_(w)
        st["w"].copy_(w)
    else:
        rnd = _mixed(counter, st["key"] ^ 0xFFFFFFFF) & 0xFFFF
        st["w"].copy_(((w.view(torch.int32) + rnd.int()) >> 16).to(torch.int16).view(torch.bfloat16))


def _adamw_state(st):
    out = {k: st[k] for k in ("w", "master", "m", "v", "m_scale", "v_scale") if k in st}
    if st["case"]["bits"] == 8:
        out["m"], out["v"] = st["m"].view(torch.float8_e4m3fn), st["v"].view(torch.float8_e4m3fn)
    return out


# ---- what the tools call

def prepare(case, seed):
    g, op = _generator(seed), case["op"]
    st = {"case": case}
    if op == "quantize":
        rows, cols = case["rows"], case["cols"]
        st["x"] = _activations(g, rows, cols)
        st["q"] = torch.empty(rows, cols, device=DEV, dtype=torch.uint8)
        st["q_t"] = torch.empty(cols, rows, device=DEV, dtype=torch.uint8)
        st["s"] = torch.empty(_pad128(cols) // 128, _pad128(rows), device=DEV, dtype=torch.uint8)
        st["s_t"] = torch.empty(_pad128(rows) // 128, _pad128(cols), device=DEV, dtype=torch.uint8)
    elif op == "gemm":
        R, C, T = case["R"], case["C"], case["T"]
        a, st["s_a"] = _plain_quantize(_activations(g, R, T), case["fmt_a"], 1)
        b, st["s_b"] = _plain_quantize(_randn(g, C, T, std=0.02).to(torch.bfloat16), case["fmt_b"], case["b_rows"])
        st["a"], st["b"] = a.view(torch.uint8), b.view(torch.uint8)
        st["c"] = _randn(g, R, C).to(torch.bfloat16)
    elif op in ("qk_fwd", "qk_bwd"):
        M, Hq, Hkv, D = case["M"], case["Hq"], case["Hkv"], case["D"]
        st["qkv"] = (_randn(g, M, (Hq + 2 * Hkv) * D) * torch.exp(_randn(g, M, 1, std=0.5))).to(torch.bfloat16)
        st["wq"], st["wk"] = ((1 + _randn(g, D, std=0.1)).to(torch.bfloat16) if case["norm"] else None for _ in range(2))
        st["positions"] = torch.randint(0, case["far"], (M,), generator=g, device=DEV)
        st["inv_freq"] = 1e6 ** (-torch.arange(0, case["rot"], 2, device=DEV, dtype=torch.float64) / case["rot"])
        st["rstd"] = torch.empty(M, Hq + Hkv, device=DEV) if case["norm"] else None
        if op == "qk_fwd":
            st["q"], st["k"] = torch.empty(M, Hq * D, device=DEV, dtype=torch.bfloat16), torch.empty(M, Hkv * D, device=DEV, dtype=torch.bfloat16)
        else:
            if case["norm"]:
                x = _heads(st["qkv"], 0, Hq + Hkv, D)
                st["rstd"] = 1.0 / torch.sqrt((x * x).mean(-1) + EPS)
            st["dq"], st["dk"], st["dv"] = (_randn(g, M, h * D, std=1e-3).to(torch.bfloat16) for h in (Hq, Hkv, Hkv))
            st["dqkv"] = torch.empty_like(st["qkv"])
            st["dwq"], st["dwk"] = (torch.empty(D, device=DEV) if case["norm"] else None for _ in range(2))
            st["amax"], st["scale"] = torch.empty(1, device=DEV), torch.empty(1, device=DEV)
        if own and op == "qk_bwd":
            from paper_2512_15306_amd import llmq
            st["ws"] = torch.empty(llmq.llmq_qk_norm_rope_workspace_bytes(M, Hq, Hkv, D), device=DEV, dtype=torch.uint8)
    else:
        matrices, vectors = _sizes(case)
        at, spans = 0, []
        for n in matrices + vectors:                     # every tensor starts at a multiple of 128 elements of its buffer
            spans.append((at, n))
            at += _pad128(n)
        there = torch.zeros(at, device=DEV, dtype=torch.bool)
        for first, n in spans:
            there[first : first + n] = True
        st["split"] = spans[len(matrices)][0]
        size = torch.exp(_randn(g, at // 128, std=1.0)).repeat_interleave(128)
        st["g"] = (_randn(g, at, std=1e-3) * size * there).to(torch.bfloat16)
        master = _randn(g, at, std=0.02) * there
        st["w"] = master.to(torch.bfloat16)
        if case["master"]:
            st["master"] = master
        m, v = _randn(g, at, std=3e-4) * size * there, (_randn(g, at, std=1e-3) * size * there) ** 2
        st["key"] = _key(STEP)
        if case["bits"] == 8:
            for name, x in (("m", m), ("v", v.sqrt())):
                b = _exponents(x.abs().view(-1, 128).amax(1), E4M3)
                st[name] = (x * _power(254 - b).repeat_interleave(128)).to(torch.float8_e4m3fn).view(torch.uint8)
                st[name + "_scale"] = b.to(torch.uint8)
        else:
            st["m"], st["v"] = m, v
        if own:
            from paper_2512_15306_amd import llmq
            part = lambda name, first, n: st[name][first : first + n] if name in st else None  # noqa: E731
            tensors = [llmq.AdamWTensor(w=part("w", a, n), master=part("master", a, n), grad=part("g", a, n), m=part("m", a, n), v=part("v", a, n),
                                        m_scale=st["m_scale"][a // 128 : (a + n + 127) // 128] if case["bits"] == 8 else None,
                                        v_scale=st["v_scale"][a // 128 : (a + n + 127) // 128] if case["bits"] == 8 else None,
                                        first_counter=a, decay=k < len(matrices), stochastic=not case["master"]) for k, (a, n) in enumerate(spans)]
            st["plan"] = llmq.llmq_adamw_plan(tensors)
    return st


def run(st):
    case = st["case"]
    op = case["op"]
    if own:
        from paper_2512_15306_amd import llmq
        if op == "quantize":
            llmq.llmq_quantize_fp8_blocks(st["x"], case["fmt"], case["block_rows"], st["q"], st["s"], st["q_t"], st["s_t"])
            return [st["q"].view(FLOAT8[case["fmt"]]), st["s"], st["q_t"].view(FLOAT8[case["fmt"]]), st["s_t"]]
        if op == "gemm":
            llmq.llmq_fp8_gemm_blocks(st["a"], st["s_a"], case["fmt_a"], st["b"], st["s_b"], case["fmt_b"], st["c"], case["accumulate"])
            return st["c"]
        if op == "qk_fwd":
            llmq.llmq_qk_norm_rope_fwd(st["qkv"], case["Hq"], case["Hkv"], case["D"], st["wq"], st["wk"], EPS, st["positions"], st["inv_freq"], case["interleaved"],
                                       st["q"], st["k"], st["rstd"])
            return [st["q"], st["k"]] + ([st["rstd"]] if case["norm"] else [])
        if op == "qk_bwd":
            llmq.llmq_qk_norm_rope_bwd(st["dq"], st["dk"], st["dv"], st["qkv"], case["Hq"], case["Hkv"], case["D"], st["wq"], st["wk"], st["rstd"], st["positions"], st["inv_freq"],
                                       case["interleaved"], st["dqkv"], st["dwq"], st["dwk"], False, E5M2, st["amax"], st["scale"], st["ws"])
            return [st["dqkv"]] + ([st["dwq"], st["dwk"]] if case["norm"] else []) + [st["amax"]]
        llmq.llmq_adamw_step(st["plan"], llmq.llmq_adamw_hyper(STEP, LR, BETA1, BETA2, DELTA, DECAY, SEED))
        return _adamw_state(st)
    if op == "quantize":
        q, s = _plain_quantize(st["x"], case["fmt"], case["block_rows"])
        q_t, s_t = _plain_quantize(st["x"].t(), case["fmt"], case["block_rows"])
        return [q, s, q_t, s_t]
    if op == "gemm":
        c = torch.matmul(_dequantized(st["a"], st["s_a"], case["fmt_a"]), _dequantized(st["b"], st["s_b"], case["fmt_b"]).t())
        st["c"].copy_(c + st["c"].float() if case["accumulate"] else c)
        return st["c"]
    if op == "qk_fwd":
        return _plain_qk_fwd(st)
    if op == "qk_bwd":
        return _plain_qk_bwd(st)
    _plain_adamw(st)
    return _adamw_state(st)


def work(case):
    op = case["op"]
    if op == "quantize":
        rows, cols = case["rows"], case["cols"]
        return {"bytes": 4 * rows * cols + rows * -(-cols // 128) + cols * -(-rows // 128), "flops": 4 * rows * cols}
    if op == "gemm":
        R, C, T = case["R"], case["C"], case["T"]
        return {"bytes": (R + C) * T + (R + C) * -(-T // 128) + (4 if case["accumulate"] else 2) * R * C, "flops": 2 * R * C * T}
    if op in ("qk_fwd", "qk_bwd"):
        M, Hq, Hkv, D = case["M"], case["Hq"], case["Hkv"], case["D"]
        x, stats = M * (Hq + Hkv) * D, M * (Hq + Hkv) if case["norm"] else 0
        if op == "qk_fwd":
            return {"bytes": 4 * x + 4 * stats + 8 * M, "flops": 10 * x}
        # the norm's gradient reads the projection again; the gradient of V is moved to its place
        return {"bytes": (6 if case["norm"] else 4) * x + 4 * stats + 4 * M * Hkv * D + 8 * M, "flops": 20 * x}
    n = sum(map(sum, _sizes(case)))
    states = 4 * (1 + 1 / 128) if case["bits"] == 8 else 16
    return {"bytes": n * (2 + states + (10 if case["master"] else 4)), "flops": 20 * n}


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
    e = _floor_log2(y.abs()).clamp(min=least)
    step = _two_to(e - mantissa_bits)
    return torch.round(y / step) * step


def _exact_codes(x, fmt, block_rows):
    largest, bits, least = (448.0, 3, -6) if fmt == E4M3 else (57344.0, 2, -14)
    rows, cols = x.shape
    y = torch.zeros(_pad128(rows), _pad128(cols), device=x.device, dtype=torch.float64)
    y[:rows, :cols] = x.double()
    y = y.view(-1, block_rows, y.shape[1] // 128, 128)
    amax = y.abs().amax((1, 3), keepdim=True)
    d = _two_to(_ceil_log2(amax / largest).clamp(min=-127))
    return _grid(y / d, bits, least).reshape(_pad128(rows), -1)[:rows, :cols]


def _exact_values(q, s, fmt):
    r = torch.arange(q.shape[0], device=q.device)
    place = (r // 128) * 128 + (r % 16) * 8 + (r % 128) // 16
    return q.view(FLOAT8[fmt]).double() * _two_to(s.double() - 127)[:, place].t().repeat_interleave(128, 1)[:, : q.shape[1]]


def _exact_turn(x, st, back):
    """Pairs of every head as complex numbers, times e^(i angle) or its conjugate."""
    c, angle = st["case"], st["positions"].double()[:, None] * st["inv_freq"][None, :]
    turn = torch.polar(torch.ones_like(angle), -angle if back else angle)[:, None, :]
    r, y = c["rot"], x.clone()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if c["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    op, st = case["op"], prepare(case, seed)
    if op == "quantize":
        x = st["x"]
        return [_exact_codes(x, case["fmt"], case["block_rows"]), None, _exact_codes(x.t(), case["fmt"], case["block_rows"]), None]
    if op == "gemm":
        c = _exact_values(st["a"], st["s_a"], case["fmt_a"]) @ _exact_values(st["b"], st["s_b"], case["fmt_b"]).t()
        return c + st["c"].double() if case["accumulate"] else c
    if op == "qk_fwd":
        M, Hq, Hkv, D = case["M"], case["Hq"], case["Hkv"], case["D"]
        x = st["qkv"].double().view(M, -1, D)[:, : Hq + Hkv]
        inverse = (x.square().mean(-1) + EPS).rsqrt()
        if case["norm"]:
            x = x * inverse[..., None] * torch.cat((st["wq"].double().expand(Hq, D), st["wk"].double().expand(Hkv, D)))
        y = _exact_turn(x, st, False)
        return [y[:, :Hq].reshape(M, -1), y[:, Hq:].reshape(M, -1)] + ([inverse] if case["norm"] else [])
    if op == "qk_bwd":
        M, Hq, Hkv, D = case["M"], case["Hq"], case["Hkv"], case["D"]
        dy = torch.cat((st["dq"], st["dk"]), 1).double().view(M, -1, D)
        dn, dws = _exact_turn(dy, st, True), []
        if case["norm"]:
            x = st["qkv"].double().view(M, -1, D)[:, : Hq + Hkv]
            r = st["rstd"].double()[..., None]
            w = torch.cat((st["wq"].double().expand(Hq, D), st["wk"].double().expand(Hkv, D)))
            dws = [(dn * x * r)[:, :Hq].sum((0, 1)), (dn * x * r)[:, Hq:].sum((0, 1))]
            dn = r * dn * w - x * r**3 * (dn * w * x).sum(-1, keepdim=True) / D
        dqkv = torch.cat((dn.reshape(M, -1), st["dv"].double()), 1)
        return [dqkv] + dws + [dqkv.abs().max().view(1).float().to(torch.bfloat16).double()]
    n, bits = st["w"].numel(), case["bits"]
    block = torch.arange(n, device=DEV) // 128
    held = lambda name: st[name].view(torch.float8_e4m3fn).double() * _two_to(st[name + "_scale"].double() - 127)[block]  # noqa: E731
    m, v = (held("m"), held("v").square()) if bits == 8 else (st["m"].double(), st["v"].double())
    g, w = st["g"].double(), (st["master"] if case["master"] else st["w"]).double()
    m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g * g
    w = w * (1 - LR * DECAY * (torch.arange(n, device=DEV) < st["split"])) - LR * (m / (1 - BETA1**STEP)) / ((v / (1 - BETA2**STEP)).sqrt() + DELTA)
    out = {"w": w}
    if case["master"]:
        out["master"] = w
    if bits == 32:
        return out | {"m": m, "v": v}
    random = _mixed(torch.arange(n, device=DEV), st["key"])
    for name, x, rnd in (("m", m, random % 65536), ("v", v.sqrt(), random // 65536)):
        amax = x.abs().view(-1, 128).amax(1)
        a = x.abs() / _two_to(_ceil_log2(amax / 448).clamp(min=-127))[block]
        step = _two_to(_floor_log2(a).clamp(min=-6) - 3)
        y = torch.where(a >= 2.0**-6, torch.floor(a / step + rnd.double() / 65536) * step, torch.round(a * 512) / 512)
        out[name] = torch.where((y == 0) & (x > 0), 2.0**-9, y) if name == "v" else y * torch.sign(x)
    return out | {"m_scale": None, "v_scale": None}
