"""Reference of the 8-bit layers in numpy, 64 bits throughout: e4m3 rounding, quantised rows, the norm, products.

Test infrastructure, never on the product path.  e4m3 here is the OCP format: 1 sign, 4 exponent and 3 mantissa bits, bias 7, largest
value 448, smallest step 2^-9, no infinities, one NaN code (0x7f, either sign).
"""
from __future__ import annotations

import math

import numpy as np

BLOCK, TOP, TINY = 128, 448.0, 2.0 ** -126


def code_values() -> np.ndarray:
    """The 256 values that the codes stand for."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v[c] = math.nan if (e, m) == (15, 7) else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        if c & 128:
            v[c] = -v[c]
    return v


def nearest(v: np.ndarray) -> np.ndarray:
    """The e4m3 value next to v (|v| < 464), ties to the one with an even mantissa."""
    v = np.asarray(v, dtype=np.float64)
    _, e = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(e - 4, -9))
    return np.clip(np.round(v / step) * step, -TOP, TOP)


def blocks(n: int) -> int:
    return -(-n // BLOCK)


def quantize_rows(v: np.ndarray):
    """(code values [R, C], scales [R, blocks]) of rows; a block with a NaN or an infinity is NaN throughout."""
    R, C = v.shape
    scales = np.empty((R, blocks(C)))
    q = np.empty((R, C))
    for b in range(blocks(C)):
        s = slice(b * BLOCK, min(C, (b + 1) * BLOCK))
        most = np.abs(v[:, s]).max(axis=1) if R else np.empty(0)
        scales[:, b] = np.where(np.isfinite(most), np.maximum(most / TOP, TINY), np.nan)
        with np.errstate(invalid="ignore"):
            q[:, s] = nearest(v[:, s] / scales[:, b:b + 1])
    return q, scales


def dequantize_rows(q: np.ndarray, scales: np.ndarray) -> np.ndarray:
    return q * np.repeat(scales, BLOCK, axis=1)[:, :q.shape[1]]


def weight_scales(w: np.ndarray) -> np.ndarray:
    N, K = w.shape
    s = np.empty((blocks(N), blocks(K)))
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            most = np.abs(w[i * BLOCK:(i + 1) * BLOCK, j * BLOCK:(j + 1) * BLOCK]).max()
            s[i, j] = max(most / TOP, TINY) if np.isfinite(most) else np.nan
    return s


def spread(scales: np.ndarray, N: int, K: int) -> np.ndarray:
    """One scale per 128 x 128 block -> one per element."""
    return np.repeat(np.repeat(scales, BLOCK, axis=0)[:N], BLOCK, axis=1)[:, :K]


def pack(codes: np.ndarray) -> np.ndarray:
    """The products' layout of one matrix of codes (uint8 [N, K]), flat."""
    N, K = codes.shape
    nb, kb = blocks(N) * 8, blocks(K)
    full = np.zeros((nb * 16, kb * BLOCK), dtype=np.uint8)
    full[:N, :K] = codes
    # (nb, r, kb, h, g, 16) -> (nb, kb, h, g, r, 16)
    return full.reshape(nb, 16, kb, 2, 4, 16).transpose(0, 2, 3, 4, 1, 5).reshape(-1)


def norm(s: np.ndarray, weight, eps: float) -> np.ndarray:
    """The norm of rows s (the rounded sum of x and the residual)."""
    n = s / np.sqrt((s * s).mean(axis=1, keepdims=True) + eps)
    return n if weight is None else n * weight


def activate(v: np.ndarray, act: str) -> np.ndarray:
    if act == "relu":
        return np.where(v < 0, 0.0, v)
    if act == "gelu":
        from scipy.special import ndtr
        return v * ndtr(v)
    return v


def linear(a, w, bias=None, act="none"):
    """(act(a w^T + bias), sum |a| |w| + |bias|): the result and what rounding errors of its sum are relative to."""
    z, size = a @ w.T, np.abs(a) @ np.abs(w).T
    if bias is not None:
        z, size = z + bias, size + np.abs(bias)
    return activate(z, act), size
