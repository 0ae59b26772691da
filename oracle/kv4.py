"""4-bit key/value cache, the attention weights its positions draw and the eviction
by them, in float64.

A code is the nearest 4-bit float (ties to even) to x / scale: sign, 2 exponent
bits of bias 1, 1 mantissa bit, largest 6, steps of 1/2 below 2.  A scale belongs to
32 neighbouring dimensions of one position: the smallest 2^e, -100 <= e <= 125, with
max|x| <= 6 2^e (2^125 where that is not enough, magnitudes then being 6 at most);
NaN where an element is not finite.
"""
import math

import numpy as np

from oracle import kv8

TABLE = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GROUP = 32
NAN_BYTE = 255


def round_to(y):
    """y rounded to the format's values, 6 at most."""
    y = np.asarray(y, dtype=np.float64)
    a = np.minimum(np.abs(y), 6.0)
    step = np.where(a < 2.0, 0.5, np.where(a < 4.0, 1.0, 2.0))
    return np.copysign(np.rint(a / step) * step, y)


def to_codes(v):
    """Codes 0..15 of values that the format has."""
    return (np.searchsorted(TABLE, np.abs(v)) + 8 * np.signbit(v)).astype(np.uint8)


def from_codes(code):
    code = np.asarray(code)
    return np.where(code & 8, -1.0, 1.0) * TABLE[code & 7]


def need(x):
    """The scale byte that an array of values needs."""
    x = np.asarray(x, dtype=np.float64)
    if not np.all(np.isfinite(x)):
        return NAN_BYTE
    e, a = -100, float(np.max(np.abs(x), initial=0.0))
    while e < 125 and a > 6.0 * 2.0 ** e:
        e += 1
    return e + 127


def scale_of(byte):
    byte = np.asarray(byte)
    return np.where(byte == NAN_BYTE, math.nan, np.ldexp(1.0, byte.astype(np.int64) - 127))


def quantise(x):
    """Values of codes and scale bytes of the last dimension's groups."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(-1, GROUP)
    fine = np.isfinite(g).all(-1)
    g = np.where(fine[:, None], g, 0.0)
    m, e = np.frexp(np.abs(g).max(-1))      # m 2^e, m in [1/2, 1); 6 = 0.75 2^3
    e = np.where(m == 0.0, -100, np.clip(e - 3 + (m > 0.75), -100, 125))
    code = round_to(g / np.ldexp(1.0, e)[:, None])
    byte = np.where(fine, e + 127, NAN_BYTE).astype(np.uint8)
    return code.reshape(x.shape), byte.reshape(*x.shape[:-1], -1)


class Cache:
    """code and scale byte of every position; shapes [n_seq, KV, 2, s_max, dh] and
    [..., s_max, dh / 32]; sums [n_seq, KV, s_max]."""

    def __init__(self, n_seq, kv_heads, dh, s_max):
        self.s_max = s_max
        self.code = np.zeros((n_seq, kv_heads, 2, s_max, dh))
        self.scale = np.full((n_seq, kv_heads, 2, s_max, dh // GROUP), 27, dtype=np.uint8)
        self.sums = np.zeros((n_seq, kv_heads, s_max))

    def store(self, x, pos):
        """x [n_seq, n, 2, KV, dh] at positions pos[b] .. of each sequence
        (None: left out)."""
        n = x.shape[1]
        for b, p in enumerate(pos):
            if p is None:
                continue
            code, byte = quantise(x[b].transpose(2, 1, 0, 3))      # [KV, 2, n, dh]
            self.code[b, :, :, p:p + n], self.scale[b, :, :, p:p + n] = code, byte
            self.sums[b, :, p:p + n] = 0.0

    def read(self):
        """Values of every position, [n_seq, KV, 2, s_max, dh]."""
        return self.code * np.repeat(scale_of(self.scale), GROUP, axis=-1)

    def pack(self, fill=0):
        """Bytes of the codes as the library lays them, positions behind s_max as
        `fill`."""
        B, KV, _, S, dh = self.code.shape
        s8 = -(-S // 8) * 8
        q = to_codes(self.code)
        keys = np.full((B, KV, s8, dh // 2), fill, dtype=np.uint8)
        keys[:, :, :S] = q[:, :, 0, :, 0::2] | q[:, :, 0, :, 1::2] << 4
        v = q[:, :, 1].reshape(B, KV, S, dh // 32, 2, 16)
        byte = np.full((B, KV, s8, dh // 32, 16), fill, dtype=np.uint8)
        byte[:, :, :S] = v[..., 0, :] | v[..., 1, :] << 4
        values = byte.reshape(B, KV, s8 // 8, 8, dh // 32, 16).transpose(0, 1, 2, 5, 4, 3)
        return np.concatenate((keys.reshape(B, KV, -1), values.reshape(B, KV, -1)), -1).reshape(-1)


def unpack(raw, n_seq, kv_heads, dh, s_max):
    """Codes 0..15 [n_seq, KV, 2, S8, dh] of a packed buffer."""
    s8 = -(-s_max // 8) * 8
    raw = np.asarray(raw, dtype=np.uint8).reshape(n_seq, kv_heads, 2, s8 * dh // 2)
    out = np.zeros((n_seq, kv_heads, 2, s8, dh), dtype=np.uint8)
    k = raw[:, :, 0].reshape(n_seq, kv_heads, s8, dh // 2)
    out[:, :, 0, :, 0::2], out[:, :, 0, :, 1::2] = k & 15, k >> 4
    v = raw[:, :, 1].reshape(n_seq, kv_heads, s8 // 8, 16, dh // 32, 8).transpose(0, 1, 2, 5, 4, 3)
    v = v.reshape(n_seq, kv_heads, s8, dh // 32, 16)
    out[:, :, 1] = np.stack((v & 15, v >> 4), -2).reshape(n_seq, kv_heads, s8, dh)
    return out


def weights(values, q, pos, alibi):
    """What each position draws: [n_seq, KV, S], the softmax weights of q [n_seq, n,
    H, dh] at positions pos[b] + j summed over a head's queries and rows."""
    B, n, H, dh = q.shape
    KV, S = values.shape[1], values.shape[3]
    m_h = kv8.slopes(H)
    out = np.zeros((B, KV, S))
    for b, p in enumerate(pos):
        if p is None:
            continue
        for h in range(H):
            for j in range(n):
                c = p + j + 1
                s = values[b, h * KV // H, 0, :c] @ q[b, j, h] / math.sqrt(dh)
                if alibi:
                    s = s - m_h[h] * (p + j - np.arange(c))
                w = np.exp(s - np.max(s))
                out[b, h * KV // H, :c] += w / np.sum(w)
    return out


def evict(sums, length, keep, recent):
    """Positions of one head that stay, ascending."""
    if length <= keep:
        return list(range(length))
    old = length - recent
    rank = [(-math.inf if math.isnan(v) else -v, not math.isnan(v), i) for i, v in enumerate(np.asarray(sums)[:old])]
    return sorted(i for _, _, i in sorted(rank)[:keep - recent]) + list(range(old, length))
