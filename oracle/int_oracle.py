"""Reference of the int8 layers and of the routing by scores in numpy, 64 bits throughout.

Test infrastructure, never on the product path.
"""
from __future__ import annotations

import numpy as np

TOP, TINY = 127.0, 2.0 ** -126
FLT_MAX = float(np.finfo(np.float32).max)


def quantize_rows(v: np.ndarray, factor=None):
    """(codes [R, C], scales [R]) of the rows v * factor [R, 1]: the whole numbers next to 127 v / max |v|, ties to even.  A row with a NaN, an
    infinity or a value beyond fp32's range has a NaN for its scale and codes of zero."""
    v = np.asarray(v, dtype=np.float64)
    R, C = v.shape
    f = np.ones((R, 1)) if factor is None else np.asarray(factor, dtype=np.float64).reshape(R, 1)
    with np.errstate(all="ignore"):
        top = np.abs(v).max(axis=1, keepdims=True) if R else np.empty((0, 1))
        most = top * f
        bad = ~(most <= FLT_MAX) | ~np.isfinite(f)
        scales = np.where(bad, np.nan, np.maximum(most / TOP, TINY))
        t = np.where(most < TOP * TINY, v * f * 2.0 ** 126, v * TOP / np.where(top > 0, top, 1.0))
        codes = np.where(bad, 0.0, np.rint(t))
    return codes.astype(np.int8), scales[:, 0]


def quantize_weights(w: np.ndarray):
    """(codes [N, K], fp32 scales [N]): the quotient by the fp32 scale is rounded to fp32 first."""
    w = np.asarray(w, dtype=np.float32)
    with np.errstate(all="ignore"):
        most = np.abs(w).max(axis=1)
        scale = np.where(np.isfinite(most), np.maximum(most / np.float32(TOP), np.float32(TINY)), np.float32(np.nan)).astype(np.float32)
        codes = np.where(np.isfinite(most)[:, None], np.rint(w / scale[:, None]), 0)
    return codes.astype(np.int8), scale


def norm_parts(s: np.ndarray, weight, eps: float):
    """(s w, 1 / rms): the norm of rows s is their product."""
    s = np.asarray(s, dtype=np.float64)
    rho = 1.0 / np.sqrt((s * s).mean(axis=1, keepdims=True) + eps)
    return s if weight is None else s * np.asarray(weight, dtype=np.float64), rho


def activate(v: np.ndarray, act: str) -> np.ndarray:
    v = np.asarray(v, dtype=np.float64)
    if act == "relu":
        return np.where(v < 0, 0.0, v)
    with np.errstate(over="ignore", invalid="ignore"):
        if act == "gelu":
            from scipy.special import erfc
            return 0.5 * v * erfc(-v * np.sqrt(0.5))
        if act == "silu":
            return v / (1.0 + np.exp(-v))
    return v


def product(a, sa, w, sw, bias=None):
    """(sa sw a w^T + bias, |sa sw a w^T|): before the activation, and what the errors of its scales are relative to.  The sums of whole numbers are
    exact: they stay below 2^53."""
    z = (a.astype(np.float64) @ w.astype(np.float64).T) * np.asarray(sa, dtype=np.float64)[:, None] * np.asarray(sw, dtype=np.float64)[None]
    return (z if bias is None else z + np.asarray(bias, dtype=np.float64)), np.abs(z)


def route(logits, k, score="softmax", balance=None, groups=1, kept=1, top=1, renormalize=False, scale=1.0):
    """(experts [T, k], weights [T, k]), token by token as the definition reads."""
    logits = np.asarray(logits, dtype=np.float64)
    T, E = logits.shape
    idx, weight = np.empty((T, k), dtype=np.int32), np.empty((T, k))
    size = E // groups
    for t in range(T):
        l = logits[t]
        invalid = bool(np.isnan(l).any() or (score == "softmax" and np.isposinf(l).any()))
        with np.errstate(all="ignore"):
            if score == "sigmoid":
                p = 1.0 / (1.0 + np.exp(-l))
            else:
                best = np.fmax.reduce(l)
                p = np.where(np.isneginf(l), 0.0, np.exp(l - best))
                p = p / p.sum()
        there = l > -np.inf                                   # not NaN, not masked
        c = np.where(there, l if balance is None else p + np.asarray(balance, dtype=np.float64), -np.inf)
        c = np.where(np.isnan(c), -np.inf, c)
        if groups > 1:
            v = np.where(there & ~np.isnan(p), p, -np.inf) if top == 2 and balance is None else c
            with np.errstate(invalid="ignore"):              # infinity and -infinity
                value = np.sort(v.reshape(groups, size), axis=1)[:, ::-1][:, :top].sum(axis=1)
            stay = np.argsort(-value, kind="stable")[:kept]
            kept_ones = np.flatnonzero(np.isin(np.arange(E) // size, stay))
        else:
            kept_ones = np.arange(E)
        order = kept_ones[np.argsort(-c[kept_ones], kind="stable")[:k]]
        w = np.where(c[order] > -np.inf, p[order], 0.0)
        if renormalize:
            w = w / w.sum() if w.sum() > 0 else np.zeros(k)
        idx[t], weight[t] = order, np.nan if invalid else w * scale
    return idx, weight
