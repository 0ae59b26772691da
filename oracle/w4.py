"""Weights in 4 bits with a scale for each group of neighbouring k, and projections
by them, in float64.

E2M1: codes and scales as the 4-bit cache's (oracle.kv4), groups of 32.  INT4:
integers -7..7 times a bfloat16 scale, max|w| / 7 rounded to nearest (ties to
even), at least 2^-100; NaN where an element is not finite.
"""
import math

import numpy as np

from oracle import kv4

E2M1, INT4 = 0, 1


def bf16(x):
    """x (float64) rounded to bfloat16, ties to even; normal numbers only."""
    m, e = np.frexp(np.asarray(x, dtype=np.float64))
    return np.ldexp(np.rint(m * 256.0), e - 8)


def quantise(fmt, group, w):
    """code values and scales (numbers) of w [n, k], k padded to whole groups."""
    w = np.asarray(w, dtype=np.float64)
    n, k = w.shape
    w = np.pad(w, ((0, 0), (0, -k % group)))
    if fmt == E2M1:
        code, byte = kv4.quantise(w)
        return code, kv4.scale_of(byte)
    g = w.reshape(n, -1, group)
    fine = np.isfinite(g).all(-1)
    g = np.where(fine[..., None], g, 0.0)
    s = np.maximum(bf16(np.abs(g).max(-1) / 7.0), 2.0 ** -100)
    code = np.clip(np.rint(g / s[..., None]), -7, 7)
    return code.reshape(n, -1), np.where(fine, s, math.nan)


def values(fmt, group, w):
    """What the 4 bits stand for, [n, k]."""
    code, s = quantise(fmt, group, w)
    return (code * np.repeat(s, group, -1))[:, :w.shape[1]]


def dwords(fmt, code):
    """The packed codes [ceil(n / 8)][ceil(k / 256)][64][4] of code values [n, k]."""
    n, k = code.shape
    T, C = -(-n // 8), -(-k // 256)
    out = np.zeros((T, C, 64, 4), dtype=np.uint32)
    q = kv4.to_codes(code) if fmt == E2M1 else (np.abs(code).astype(np.uint8) | np.signbit(code) * 8 * (code != 0))
    for i in range(n):
        for j in range(k):
            h, s, g, e = j // 128 % 2, j // 32 % 4, j // 8 % 4, j % 8
            c = int(q[i, j])
            if fmt == E2M1:
                bits = c << (4 * e)
            elif e < 4:
                bits = (c & 7) << (8 * e) | (c >> 3) << (8 * e + 7)
            else:
                bits = (c & 7) << (8 * (e - 4) + 4) | (c >> 3) << ((8 * (e - 4) + 11) % 32)
            out[i // 8, j // 256, 16 * g + 8 * h + i % 8, s] |= bits
    return out


def project(x, w, g=None, eps=1e-5, alpha=1.0, R=None, act="none"):
    """act(R + alpha x' w^T), x' the RMSNorm of x's rows with gain g."""
    if g is not None:
        x = x / np.sqrt(np.mean(x ** 2, -1, keepdims=True) + eps) * g
    y = alpha * (x @ w.T)
    if act == "swiglu":
        u, v = np.split(y, 2, -1)
        return u / (1.0 + np.exp(-u)) * v
    if act == "relu2":
        return np.maximum(y, 0.0) ** 2
    return y if R is None else y + R
