"""Layer normalisation, 8-bit block tensors, GeLU's gradient and products of 8-bit tensors in 64 bits, from their definitions (numpy).

An 8-bit number is decoded from its bits and encoded by search over all of the type's values, so that neither shares a step with any
conversion instruction.  A block is 128 consecutive values of a stored row; its scale 2^e has e the smallest integer >= -127 with
max|block| / 2^e within the type, the maximum over finite values.
"""
from __future__ import annotations

import numpy as np
from scipy.special import erfc

BLOCK = 128
#: (exponent bits, bias, fraction bits)
FORMATS = {"e4m3": (4, 7, 3), "e5m2": (5, 15, 2)}


def decode_table(kind: str) -> np.ndarray:
    """The 256 values of the type: e4m3 has one NaN a sign and no infinity, e5m2 IEEE-like specials."""
    eb, bias, fb = FORMATS[kind]
    out = np.empty(256)
    for code in range(256):
        sign = -1.0 if code & 0x80 else 1.0
        e, f = (code >> fb) & ((1 << eb) - 1), code & ((1 << fb) - 1)
        if kind == "e4m3" and (code & 0x7F) == 0x7F:
            v = np.nan
        elif kind == "e5m2" and e == 31:
            v = np.inf if f == 0 else np.nan
        elif e == 0:
            v = f * 2.0 ** (1 - bias - fb)
        else:
            v = (1 + f / (1 << fb)) * 2.0 ** (e - bias)
        out[code] = sign * v
    return out


def largest(kind: str) -> float:
    t = decode_table(kind)
    return float(t[np.isfinite(t)].max())


def encode(x: np.ndarray, kind: str) -> np.ndarray:
    """Codes of the nearest values, ties to the even code; |x| within the type."""
    table = decode_table(kind)[:128]
    n = int(np.isfinite(table).sum())
    mag = table[:n]
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    assert (a <= mag[-1]).all()
    hi = np.clip(np.searchsorted(mag, a, side="left"), 0, n - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = mag[hi] - a, a - mag[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    code = np.where(np.isinf(x), 0x7C if kind == "e5m2" else 0x7F, code)
    code = np.where(np.isnan(x), 0x7F, code)
    return (code + np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def scale_bytes(x: np.ndarray, kind: str) -> np.ndarray:
    """x [rows, n] -> bytes [rows, ceil(n / 128)]"""
    rows, n = x.shape
    nb = -(-n // BLOCK)
    out = np.empty((rows, nb), np.uint8)
    top = largest(kind)
    for b in range(nb):
        part = np.abs(x[:, b * BLOCK:(b + 1) * BLOCK])
        most = np.where(np.isfinite(part), part, 0.0).max(1)
        for r in range(rows):
            e = -127
            if most[r] > 0:
                e = max(-127, int(np.floor(np.log2(most[r]))) - 18)   # below it, then up
                while most[r] / 2.0 ** e > top:
                    e += 1
            out[r, b] = e + 127
    return out


def spread(scales: np.ndarray, n: int) -> np.ndarray:
    """2^e for every value of rows of n"""
    return np.repeat(2.0 ** (scales.astype(np.float64) - 127), BLOCK, axis=1)[:, :n]


def quantize(x: np.ndarray, kind: str):
    s = scale_bytes(x, kind)
    return encode(x / spread(s, x.shape[1]), kind), s


def dequantize(q: np.ndarray, s: np.ndarray, kind: str) -> np.ndarray:
    return decode_table(kind)[q] * spread(s, q.shape[1])


def gelu(x):
    return 0.5 * x * erfc(-x / np.sqrt(2.0))


def gelu_slope(x):
    return 0.5 * erfc(-x / np.sqrt(2.0)) + x * np.exp(-0.5 * x * x) / np.sqrt(2.0 * np.pi)


def layernorm(x, gamma, beta, eps):
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    xhat = (x - mean[:, None]) * rstd[:, None]
    return xhat * gamma + beta, mean, rstd


def layernorm_grad(x, gamma, mean, rstd, dy):
    xhat = (x - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xhat * (g * xhat).mean(1, keepdims=True))
    return dx, (dy * xhat).sum(0), dy.sum(0)
