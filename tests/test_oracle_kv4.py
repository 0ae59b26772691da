"""The 4-bit cache's, weights' and eviction's oracles against their definitions."""
import math

import numpy as np
import pytest

from oracle import kv4, kv8, w4


def test_rounding_is_the_nearest():
    """Every bf16 between -7 and 7, against a search through the sixteen values."""
    y = (np.arange(0x40E1, dtype=np.uint32) << 16).view(np.float32).astype(np.float64)     # 0 to 7
    y = y[np.isfinite(y) & (y <= 7)]
    y = np.concatenate((y, -y))
    got = kv4.round_to(y)
    far = np.abs(np.abs(y)[:, None] - kv4.TABLE)
    best = far.min(1)
    assert np.array_equal(np.abs(np.abs(y) - np.abs(got)), best)
    # ties: the even code
    tie = (far == best[:, None]).sum(1) == 2
    assert tie.any() and np.all(kv4.to_codes(got)[tie] % 2 == 0)
    assert np.array_equal(np.signbit(got), np.signbit(y))


def test_codes_and_values():
    c = np.arange(16)
    assert np.array_equal(kv4.to_codes(kv4.from_codes(c))[1:], c[1:])
    assert kv4.from_codes(7) == 6 and kv4.from_codes(15) == -6 and kv4.from_codes(1) == 0.5


@pytest.mark.parametrize("a,e", [(6.0, 0), (6.03125, 1), (3.0, -1), (3.015625, 0), (0.0, -100), (2.0 ** -140, -100),
                                 (6 * 2.0 ** 125, 125), (3.3895e38, 125), (math.inf, None), (math.nan, None)])
def test_scale(a, e):
    x = np.zeros(32)
    x[7] = -a
    assert kv4.need(x) == (255 if e is None else e + 127) == kv4.quantise(x)[1][0]


@pytest.mark.parametrize("dh", [64, 128])
def test_pack_and_unpack(dh):
    rng = np.random.default_rng(dh)
    c = kv4.Cache(2, 3, dh, 21)
    c.store(rng.standard_normal((2, 17, 2, 3, dh)), [0, 4])
    raw = kv4.unpack(c.pack(fill=0xEE), 2, 3, dh, 21)
    assert np.array_equal(kv4.from_codes(raw[..., :21, :]), c.code)
    assert np.all(raw[..., 21:, :] == 14)
    # one byte by its place in the header's words: sequence 1, head 2, position 13, dimensions 33 and 49
    s8, b, h, p, i, j = 24, 1, 2, 13, 1, 1
    at = (b * 3 + h) * s8 * dh + s8 * dh // 2 + ((p // 8 * 16 + i) * (dh // 32) + j) * 8 + p % 8
    v = kv4.to_codes(c.code[b, h, 1, p])
    assert c.pack()[at] == v[32 * j + i] | v[32 * j + 16 + i] << 4
    at = (b * 3 + h) * s8 * dh + p * dh // 2 + 5
    k = kv4.to_codes(c.code[b, h, 0, p])
    assert c.pack()[at] == k[10] | k[11] << 4


def test_rows_do_not_touch_each_other():
    rng = np.random.default_rng(1)
    a, b = kv4.Cache(1, 1, 64, 20), kv4.Cache(1, 1, 64, 20)
    x = rng.standard_normal((1, 20, 2, 1, 64))
    a.store(x, [0])
    b.store(x[:, :9], [0])
    b.store(1e6 * x[:, 9:12], [9])      # a draft, taken back
    for i in range(9, 20):
        b.store(x[:, i:i + 1], [i])
    assert np.array_equal(a.code, b.code) and np.array_equal(a.scale, b.scale)


def test_weights_sum_to_the_rows():
    rng = np.random.default_rng(2)
    v = rng.standard_normal((2, 2, 2, 30, 64))
    q = rng.standard_normal((2, 3, 4, 64))
    w = kv4.weights(v, q, [5, None], 1)
    assert np.allclose(w[0].sum(-1), 2 * 3) and not w[1].any() and not w[0, :, 8:].any()
    # the attention's output is those weights' where there is one row and one query head
    o, _, _ = kv8.attention(v[:1, :1], q[:1, :1, :1], [20], 0)
    assert np.allclose(kv4.weights(v[:1, :1], q[:1, :1, :1], [20], 0)[0, 0] @ v[0, 0, 1], o[0, 0, 0])


def test_evict():
    s = np.array([1, 5, 0, 5, 5, 2, 9, 9.0])
    assert kv4.evict(s, 8, 4, 1) == [1, 3, 6, 7]
    assert kv4.evict(s, 8, 4, 4) == [4, 5, 6, 7]
    assert kv4.evict(s, 8, 3, 0) == [1, 6, 7]
    assert kv4.evict(s, 3, 4, 1) == [0, 1, 2] and kv4.evict(s, 0, 4, 1) == []
    assert kv4.evict(np.array([math.inf, math.nan, 3, math.nan]), 4, 2, 0) == [1, 3]
    assert kv4.evict(np.zeros(6), 6, 3, 1) == [0, 1, 5]


def test_bf16():
    import torch
    x = np.random.default_rng(0).standard_normal(4000) * 10.0 ** np.random.default_rng(1).integers(-20, 20, 4000)
    assert np.array_equal(w4.bf16(x.astype(np.float32).astype(np.float64)),
                          torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).double().numpy())


@pytest.mark.parametrize("group", [32, 64, 128])
def test_int4(group):
    rng = np.random.default_rng(group)
    w = w4.bf16(rng.standard_normal((3, 200)) * 0.02)
    code, s = w4.quantise(w4.INT4, group, w)
    assert code.shape == (3, -(-200 // group) * group) and np.abs(code).max() == 7
    v = w4.values(w4.INT4, group, w)
    assert np.all(np.abs(v - w) <= 0.5 * np.repeat(s, group, -1)[:, :200] * (1 + 2.0 ** -6))
    w[1, 70] = math.nan
    v = w4.values(w4.INT4, group, w)
    g = 70 // group
    assert np.isnan(v[1, g * group:(g + 1) * group]).all() and np.isnan(v).sum() == min(group, 200 - g * group)
    assert not w4.values(w4.INT4, group, np.zeros((1, 64))).any()


def test_dwords():
    """Bits by the header's words, for one element of each half of a dword."""
    for fmt, e, val, bits in ((w4.E2M1, 3, -1.5, (3 | 8) << 12), (w4.INT4, 2, -5, 5 << 16 | 1 << 23),
                              (w4.INT4, 7, -6, 6 << 28 | 1 << 3), (w4.INT4, 5, 7, 7 << 12)):
        code = np.zeros((12, 400))
        r, h, s, g = 3, 0, 1, 2
        code[8 + r, 256 + 128 * h + 32 * s + 8 * g + e] = val
        d = w4.dwords(fmt, code)
        assert d.shape == (2, 2, 64, 4) and d[1, 1, 16 * g + 8 * h + r, s] == bits and np.count_nonzero(d) == 1
