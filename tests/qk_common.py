"""The norm and rotation of query and key heads in binary64 on the CPU, and their gradient, from the formulas."""
import numpy as np


def columns(D, rot, interleaved):
    """Columns a and b of the turned pairs."""
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def angles(positions, inv_freq):
    """[M, 1, pairs] in extended precision, brought into one turn."""
    t = positions.astype(np.longdouble)[:, None] * inv_freq.astype(np.longdouble)[None, :]
    two_pi = np.longdouble("6.283185307179586476925286766559")
    return np.asarray(t - np.floor(t / two_pi) * two_pi, dtype=np.float64)[:, None, :]


def turned(x, angle, rot, interleaved):
    y = x.copy()
    a, b = columns(x.shape[-1], rot, interleaved)
    y[..., a] = x[..., a] * np.cos(angle) - x[..., b] * np.sin(angle)
    y[..., b] = x[..., b] * np.cos(angle) + x[..., a] * np.sin(angle)
    return y


def forward(x, w, eps, angle, rot, interleaved):
    """x [M, H, D], w [H, D] or None -> (y, rstd or None, n)."""
    if w is None:
        return turned(x, angle, rot, interleaved), None, x
    rstd = 1.0 / np.sqrt((x * x).mean(-1) + eps)
    n = x * rstd[..., None] * w
    return turned(n, angle, rot, interleaved), rstd, n


def backward(dy, x, w, rstd, angle, rot, interleaved):
    """-> (dx, terms of dw [M, H, D] or None, g)."""
    g = turned(dy, -angle, rot, interleaved)
    if w is None:
        return g, None, g
    n = x * rstd[..., None]
    a = g * w
    return rstd[..., None] * (a - n * (a * n).mean(-1, keepdims=True)), g * n, g


def of_pairs(x, rot, interleaved):
    """|x_a| + |x_b| of every column's pair (|x| behind the turned ones): what the rounding of a turned value goes by."""
    y = np.abs(x).copy()
    a, b = columns(x.shape[-1], rot, interleaved)
    y[..., a] = y[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y
