"""One AdamW step in numpy on the CPU: operation by operation in binary32, and by the formula in binary64."""
import math

import numpy as np

from tests.blocks_common import scale_code

f32 = np.float32


def bf16_values(bits):
    return (bits.astype(np.uint32) << 16).view(f32)


def bf16_bits(x):
    """To nearest even (finite values)."""
    b = x.view(np.uint32).astype(np.uint64)
    return ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)


def mixed(counter, key):
    x = (np.asarray(counter, dtype=np.uint64) * np.uint64(0x9E3779B1) + np.uint64(key)) & np.uint64(0xFFFFFFFF)
    x = (x ^ (x >> np.uint64(16))) * np.uint64(0x6A09E667) & np.uint64(0xFFFFFFFF)
    x = (x ^ (x >> np.uint64(15))) * np.uint64(0xBB67AE85) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def step_key(step, seed):
    return int(mixed(np.uint64(step), int(mixed(np.uint64(seed), 0))))


def e4m3_values(codes):
    c = codes.astype(np.int64) & 127
    v = np.where(c < 8, c * 2.0 ** -9, (8 + c % 8) * np.exp2(c // 8 - 10.0))
    return np.where(codes >= 128, -v, v)


def powers(bytes_, n):
    return np.repeat(np.exp2(bytes_.astype(np.float64) - 127), 128)[:n].astype(f32)


def codes_of(x, rnd, square, root=False):
    """(codes of the magnitudes, scale bytes) of binary32 values in blocks of 128.  square: the mean of a code's square is kept, of roots below 2^-6 always."""
    n = x.size
    blocks = np.abs(np.pad(x, (0, -n % 128))).reshape(-1, 128)
    b = np.array([scale_code(float(v), 0) for v in blocks.max(1)])
    a = (blocks.astype(np.float64) * np.exp2(127.0 - b)[:, None]).reshape(-1)[:n].astype(f32)
    small = a < 2.0 ** -6
    # the code and 20 bits behind it, of a normal value its exponent and mantissa, below 2^-6 steps of 2^-9
    at = np.where(small, np.rint(a.astype(np.float64) * 2.0 ** 29).astype(np.int64), a.view(np.uint32).astype(np.int64) - (960 << 20))
    f, unit = (at & 0xFFFFF).astype(f32) * f32(2.0 ** -20), (2 * np.where(small, at >> 20, 8 + ((at >> 20) & 7))).astype(f32)
    up = (rnd.astype(f32) + f32(0.5)) * (unit + f32(1)) < f * (unit + f) * f32(65536)
    return np.where(square | (root & small), (at >> 20) + up, (at + (rnd.astype(np.int64) << 4)) >> 20), b


class State:
    """Weights and moments of one tensor: w (BF16 bits) and master (binary32) or either alone, moments as binary32 arrays or codes and scale bytes."""

    def __init__(self, w, master, m, v, m_scale=None, v_scale=None):
        self.w, self.master, self.m, self.v, self.m_scale, self.v_scale = w, master, m, v, m_scale, v_scale

    def moments(self):
        """m and v in binary32."""
        if self.m_scale is None:
            return self.m.copy(), self.v.copy()
        n = self.m.size
        r = e4m3_values(self.v).astype(f32) * powers(self.v_scale, n)
        return e4m3_values(self.m).astype(f32) * powers(self.m_scale, n), r * r

    def weights(self):
        return self.master.copy() if self.master is not None else bf16_values(self.w)


def step_exact(state, g, t, lr, b1, b2, eps, wd, scale=1.0, decay=True):
    """(w, m, v) in binary64."""
    m, v = (x.astype(np.float64) for x in state.moments())
    w, g = state.weights().astype(np.float64), g.astype(np.float64) * scale
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    return w * (1 - lr * wd * decay) - lr * (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + eps), m, v


def step_as_rounded(state, g, t, lr, b1, b2, eps, wd, seed=0, scale=1.0, decay=True, stochastic=False, first=0):
    """The state after a step, bit for bit."""
    m, v = state.moments()
    w, g = state.weights(), g.astype(f32) * f32(scale)
    m = m * f32(b1) + g * f32(1 - b1)
    v = v * f32(b2) + (g * g) * f32(1 - b2)
    root = np.sqrt(v)
    w = (w - w * f32(lr * wd if decay else 0.0)) - (m / (root * f32(1 / math.sqrt(1 - b2 ** t)) + f32(eps))) * f32(lr / (1 - b1 ** t))
    counter, key = np.arange(g.size, dtype=np.uint64) + np.uint64(first), step_key(t, seed)
    out = State(None, None, m, v)
    if state.m_scale is not None:
        rnd = mixed(counter, key)
        mc, out.m_scale = codes_of(m, rnd & np.uint64(0xFFFF), False)
        vc, out.v_scale = codes_of(root, rnd >> np.uint64(16), b2 > 0.96875, True)
        out.m, out.v = np.where(m < 0, mc | 128, mc).astype(np.uint8), np.where((vc == 0) & (root > 0), 1, vc).astype(np.uint8)
    out.master = w if state.master is not None else None
    if state.w is not None:
        if stochastic:
            out.w = ((w.view(np.uint32).astype(np.uint64) + (mixed(counter, key ^ 0xFFFFFFFF) & np.uint64(0xFFFF))) >> np.uint64(16)).astype(np.uint16)
        else:
            out.w = bf16_bits(w)
    return out
