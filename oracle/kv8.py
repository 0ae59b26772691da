"""8-bit key/value cache and attention over it, in float64.

A code is the nearest value (ties to even) of the format to x / scale; e4m3:
sign, 4 exponent bits of bias 7, 3 mantissa bits, largest 448, steps of 2^-9
below 2^-6; int8: integers of magnitude up to 127.  A scale belongs to a block of
positions of one head's keys or values: the smallest 2^e >= 2^-100 with
max|x| <= Q 2^e, NaN where an element is not finite.  A block's scale is set when
its first position is written and only rises until that is written again; when it
rises, what the block holds is rounded again.
"""
import math

import numpy as np

E4M3, INT8 = 0, 1
QMAX = {E4M3: 448.0, INT8: 127.0}
MIN_SCALE = 2.0 ** -100


def round_to(fmt, y):
    """y rounded to the format's values (|y| <= Q)."""
    y = np.asarray(y, dtype=np.float64)
    if fmt == INT8:
        return np.rint(y)
    _, e = np.frexp(np.maximum(np.abs(y), 2.0 ** -6))   # |y| < 2^e <= 2 |y|
    step = np.ldexp(1.0, e - 4)
    return np.rint(y / step) * step


def e4m3_table():
    """The value of every byte (NaN for 0x7f and 0xff)."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = math.nan if e == 15 and m == 7 else (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
        out[c] = -v if c & 128 else v
    return out


def to_bytes(fmt, y):
    """Bytes of values that the format has (-0 as the sign bit alone in e4m3)."""
    y = np.asarray(y, dtype=np.float64)
    if fmt == INT8:
        return y.astype(np.int64).astype(np.uint8)
    pos = np.searchsorted(e4m3_table()[:127], np.abs(y)).astype(np.uint8)
    return pos | (np.signbit(y).astype(np.uint8) << 7)


def need(fmt, x):
    """The scale that an array of values needs."""
    x = np.asarray(x, dtype=np.float64)
    if not np.all(np.isfinite(x)):
        return math.nan
    s, a = MIN_SCALE, float(np.max(np.abs(x), initial=0.0))
    while a > QMAX[fmt] * s:
        s *= 2.0
    return s


class Cache:
    """code and scale of every position; shapes [n_seq, KV, 2, s_max, dh] and
    [n_seq, KV, 2, blocks]."""

    def __init__(self, fmt, block, n_seq, kv_heads, dh, s_max):
        self.fmt, self.block, self.s_max = fmt, block, s_max
        self.code = np.zeros((n_seq, kv_heads, 2, s_max, dh))
        self.scale = np.zeros((n_seq, kv_heads, 2, -(-s_max // block)))

    def store(self, x, pos):
        """x [n_seq, n, 2, KV, dh] at positions pos[b] .. of each sequence
        (None: left out)."""
        n = x.shape[1]
        for b, p in enumerate(pos):
            if p is None:
                continue
            for h in range(x.shape[3]):
                for part in range(2):
                    self._store(b, h, part, x[b, :, part, h], p, p + n)

    def _store(self, b, h, part, x, lo, hi):
        code, scale = self.code[b, h, part], self.scale[b, h, part]
        for blk in range(lo // self.block, (hi - 1) // self.block + 1):
            first = blk * self.block
            i, j = max(first, lo), min(first + self.block, hi)
            s = need(self.fmt, x[i - lo:j - lo])
            if first < lo:
                old = scale[blk]
                s = math.nan if math.isnan(old) or math.isnan(s) else max(old, s)
                if s > old:
                    code[first:lo] = round_to(self.fmt, code[first:lo] * (old / s))
            scale[blk] = s
            code[i:j] = 0.0 if math.isnan(s) else round_to(self.fmt, x[i - lo:j - lo] / s)

    def read(self):
        """Values of every position, [n_seq, KV, 2, s_max, dh]."""
        return self.code * np.repeat(self.scale, self.block, axis=-1)[..., :self.s_max, None]

    def pack(self, fill=0):
        """Bytes of the codes as the library lays them, padding as `fill`."""
        B, KV, _, S, dh = self.code.shape
        s16 = -(-S // 16) * 16
        q = np.full((B, KV, 2, s16, dh), fill, dtype=np.uint8)
        q[..., :S, :] = to_bytes(self.fmt, self.code)
        keys = q[:, :, 0].reshape(B, KV, -1)
        values = q[:, :, 1].reshape(B, KV, s16 // 16, 16, dh).transpose(0, 1, 2, 4, 3).reshape(B, KV, -1)
        return np.concatenate((keys[:, :, None], values[:, :, None]), axis=2).reshape(-1)


def unpack(raw, n_seq, kv_heads, dh, s_max):
    """Bytes [n_seq, KV, 2, s_max, dh] of a packed buffer."""
    s16 = -(-s_max // 16) * 16
    q = np.asarray(raw, dtype=np.uint8).reshape(n_seq, kv_heads, 2, s16 * dh)
    keys = q[:, :, 0].reshape(n_seq, kv_heads, s16, dh)
    values = q[:, :, 1].reshape(n_seq, kv_heads, s16 // 16, dh, 16).swapaxes(-1, -2).reshape(keys.shape)
    return np.stack((keys, values), axis=2)[..., :s_max, :]


def slopes(heads):
    """ALiBi slopes (Press et al. 2022, section 3)."""
    n = 2 ** int(math.floor(math.log2(heads)))
    return [2.0 ** (-8.0 * (h + 1) / n) if h < n else 2.0 ** (-4.0 * (2 * (h - n) + 1) / n) for h in range(heads)]


def attention(values, q, pos, alibi):
    """q [n_seq, n, H, dh] at positions pos[b] + j over values [n_seq, KV, 2,
    S, dh] of positions 0 .. pos[b] + j; query head h reads head h KV // H.
    Returns the output and, for error bounds, per row sum_k p_k |v_k| and the
    largest sum_d |q_d k_d| / sqrt(dh), ALiBi distance term and |score - max|
    of any weight that counts."""
    B, n, H, dh = q.shape
    KV = values.shape[1]
    m_h = slopes(H)
    o, a = np.zeros(q.shape), np.zeros(q.shape)
    mag = np.zeros((B, n, H, 3))
    for b, p in enumerate(pos):
        if p is None:
            continue
        for h in range(H):
            k, v = values[b, h * KV // H]
            for j in range(n):
                c = p + j + 1
                s = k[:c] @ q[b, j, h] / math.sqrt(dh)
                bias = m_h[h] * (p + j - np.arange(c)) if alibi else np.zeros(c)
                s = s - bias
                w = np.exp(s - np.max(s))
                w /= np.sum(w)
                o[b, j, h] = w @ v[:c]
                a[b, j, h] = w @ np.abs(v[:c])
                seen = w > 1e-12
                if np.any(seen):
                    mag[b, j, h] = (np.max((np.abs(k[:c]) @ np.abs(q[b, j, h]))[seen]) / math.sqrt(dh),
                                    np.max(bias[seen]), np.max(np.max(s) - s[seen]))
    return o, a, mag
