"""Plain forms of the block formats in binary64 on the CPU, for the tests: codes and scales of blocks of 128, and where a scale's byte is kept."""
import numpy as np
import torch

FLOAT8 = {0: torch.float8_e4m3fn, 1: torch.float8_e5m2}
LARGEST = {0: 448.0, 1: 57344.0}


def padded(n: int) -> int:
    return (n + 127) // 128 * 128


def scale_places(rows: int, steps: int) -> np.ndarray:
    """[rows, steps] -> index of the byte."""
    r, k = np.arange(rows)[:, None], np.arange(steps)[None, :]
    return k * padded(rows) + 128 * (r // 128) + 8 * (r % 16) + (r // 16) % 8


def scale_bytes(s: torch.Tensor, rows: int, cols: int) -> np.ndarray:
    """The scale bytes [rows, steps] of an operand."""
    return s.detach().cpu().numpy().reshape(-1)[scale_places(rows, padded(cols) // 128)].astype(np.int64)


def packed(b: np.ndarray) -> torch.Tensor:
    """Scale bytes [rows, steps] as they are kept; bytes of rows that do not exist hold rubbish."""
    rows, steps = b.shape
    out = np.full(padded(rows) * steps, 0xFF, dtype=np.uint8)
    out[scale_places(rows, steps)] = b
    return torch.from_numpy(out)


def scale_code(amax: float, fmt: int) -> int:
    """127 + the least e with amax <= LARGEST 2^e, by trying."""
    if not np.isfinite(amax):
        return 255
    if amax == 0:
        return 127
    e = -127
    while amax > LARGEST[fmt] * 2.0 ** e:
        e += 1
    return e + 127


def decode(q: torch.Tensor, fmt: int) -> np.ndarray:
    return q.detach().cpu().view(FLOAT8[fmt]).to(torch.float64).numpy()


def quantize(x: torch.Tensor, fmt: int, block_rows: int):
    """(values of the codes [rows, cols], scale bytes [rows, steps]) of a BF16 tensor."""
    v = x.detach().cpu().to(torch.float64).numpy()
    rows, cols = v.shape
    steps = padded(cols) // 128
    codes, b = np.zeros((rows, cols)), np.zeros((rows, steps), dtype=np.int64)
    mantissa, least = (3, -6) if fmt == 0 else (2, -14)
    for r in range(0, rows, block_rows):
        for k in range(steps):
            at = np.s_[r : r + block_rows, 128 * k : 128 * k + 128]
            block = v[at]
            b[r : r + block_rows, k] = code = scale_code(np.abs(block).max(), fmt)
            if code == 255:
                codes[at] = np.nan
                continue
            y = np.ldexp(block, 127 - code)
            step = np.ldexp(1.0, np.maximum(np.frexp(y)[1] - 1, least) - mantissa)
            codes[at] = np.rint(y / step) * step
    return codes, b


def values(codes: np.ndarray, b: np.ndarray) -> np.ndarray:
    """What codes (their values) and scale bytes stand for."""
    return codes * np.repeat(np.ldexp(1.0, b - 127), 128, axis=1)[:, : codes.shape[1]]
