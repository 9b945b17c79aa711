"""Products of a linear layer with narrow operands in the oracle: 8-bit floats under power-of-two block scales, the gated unit and
its gradient, in binary64.

TEST INFRASTRUCTURE ONLY; shares no code with the HIP library.

Formats: E4M3 without infinities (bias 7, largest number 448, magnitude code 127 = NaN) and E5M2 with them (bias 15, largest number
57344, codes 124 = infinity, 125..127 = NaN).  A block's scale is 2^e with the smallest integer e for which no finite element exceeds the
largest number, at least -126, 0 for a block without a non-zero finite element; its byte is e + 127.
"""
from __future__ import annotations

import numpy as np

TOP = {"E4M3": 448.0, "E5M2": 57344.0}
MANT = {"E4M3": 3, "E5M2": 2}
LEAST = {"E4M3": -6, "E5M2": -14}


def code_values(fmt: str) -> np.ndarray:
    """The 128 magnitudes by code; NaN and infinity where the format has them."""
    y, least = MANT[fmt], LEAST[fmt]
    out = np.empty(128)
    for q in range(128):
        e, f = q >> y, q & ((1 << y) - 1)
        out[q] = f * 2.0 ** (least - y) if e == 0 else (1 + f / 2 ** y) * 2.0 ** (e - 1 + least)
    if fmt == "E4M3":
        out[127] = np.nan
    else:
        out[124], out[125:] = np.inf, np.nan
    return out


def decode(codes: np.ndarray, fmt: str) -> np.ndarray:
    v = code_values(fmt)[codes & 127]
    return np.where(codes & 128, -v, v)


def encode(v: np.ndarray, fmt: str) -> np.ndarray:
    """Nearest code of |v| <= TOP, infinities and NaN; ties to the even code."""
    vals = code_values(fmt)
    n = int(np.flatnonzero(vals == TOP[fmt])[0]) + 1
    a = np.abs(v)
    hi = np.clip(np.searchsorted(vals[:n], a, side="left"), 1, n - 1)
    lo = hi - 1
    dl, dh = a - vals[lo], vals[hi] - a
    q = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    q = np.where(np.isinf(a), 127 if fmt == "E4M3" else 124, np.where(np.isnan(a), 127, q))
    return (q | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def block_exponents(x: np.ndarray, rows: int, fmt: str) -> np.ndarray:
    M, K = x.shape
    R, B = -(-M // rows), -(-K // 128)
    e = np.zeros((R, B), dtype=np.int64)
    for i in range(R):
        for j in range(B):
            b = np.abs(x[i * rows:(i + 1) * rows, j * 128:(j + 1) * 128].astype(np.float64))
            b = b[np.isfinite(b)]
            a = b.max() if b.size else 0.0
            if a > 0:
                t = int(np.floor(np.log2(a / TOP[fmt]))) - 1
                while a > TOP[fmt] * 2.0 ** t:
                    t += 1
                e[i, j] = max(t, -126)
    return e


def spread(e: np.ndarray, rows: int, M: int, K: int) -> np.ndarray:
    return np.repeat(np.repeat(e, rows, axis=0)[:M], 128, axis=1)[:, :K]


def quantize(x: np.ndarray, rows: int, fmt: str):
    """(codes uint8 [M, K], scale bytes uint8)."""
    M, K = x.shape
    e = block_exponents(x, rows, fmt)
    return encode(x.astype(np.float64) * 2.0 ** -spread(e, rows, M, K).astype(np.float64), fmt), (e + 127).astype(np.uint8)


def values(codes: np.ndarray, scales: np.ndarray, rows: int, fmt: str) -> np.ndarray:
    M, K = codes.shape
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return decode(codes, fmt) * spread(s, rows, M, K)


def silu_mul(g: np.ndarray, u: np.ndarray) -> np.ndarray:
    return g / (1 + np.exp(-g)) * u


def silu_mul_grad(g: np.ndarray, u: np.ndarray, dh: np.ndarray):
    s = 1 / (1 + np.exp(-g))
    return dh * u * s * (1 + g * (1 - s)), dh * g * s
