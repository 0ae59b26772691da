"""The 8-bit cache's oracle against torch's float8 conversion, brute force over
every code and scale, and torch attention in float64 (no GPU)."""
import math

import numpy as np
import pytest
import torch

from oracle import kv8


def test_e4m3_rounding_is_torchs():
    rng = np.random.default_rng(0)
    t = kv8.e4m3_table()
    y = np.concatenate((rng.uniform(-448, 448, 20000), rng.standard_normal(20000) * 2.0 ** -6,
                        t[np.isfinite(t)], (t[:126] + t[1:127]) / 2))          # every value, every tie
    want = torch.from_numpy(y).float()
    y = want.double().numpy()
    want = want.to(torch.float8_e4m3fn)
    got = kv8.round_to(kv8.E4M3, y)
    assert np.array_equal(got, want.double().numpy())
    assert np.array_equal(kv8.to_bytes(kv8.E4M3, got), want.view(torch.uint8).numpy())


def test_int8_rounding():
    y = np.array([-127.0, -126.5, -0.5, 0.5, 1.5, 2.5, 126.49, 127.0])
    assert np.array_equal(kv8.round_to(kv8.INT8, y), [-127, -126, 0, 0, 2, 2, 126, 127])
    assert list(kv8.to_bytes(kv8.INT8, [-127.0, -1.0, 0.0, 127.0])) == [129, 255, 0, 127]


@pytest.mark.parametrize("fmt", [kv8.E4M3, kv8.INT8])
def test_scale_is_the_smallest_power_that_fits(fmt):
    q = kv8.QMAX[fmt]
    for e in (-99, -20, 0, 3, 119):
        s = 2.0 ** e
        assert kv8.need(fmt, [q * s]) == s
        assert kv8.need(fmt, [-np.nextafter(q * s, math.inf)]) == 2 * s
    assert kv8.need(fmt, [0.0]) == kv8.need(fmt, [1e-40]) == 2.0 ** -100
    assert math.isnan(kv8.need(fmt, [1.0, math.inf])) and math.isnan(kv8.need(fmt, [math.nan]))


@pytest.mark.parametrize("fmt", [kv8.E4M3, kv8.INT8])
@pytest.mark.parametrize("block", [16, 128])
def test_store_in_pieces(fmt, block):
    """Rows written one call or several: within a step of the values, and bit
    equal where the block's scale is set by its first piece."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((2, 150, 2, 3, 8))
    x[:, ::block] *= 4.0          # the first row of every block sets its scale
    one, many = (kv8.Cache(fmt, block, 2, 3, 8, 160) for _ in range(2))
    one.store(x, [5, 0])
    assert np.any(one.read()[1] != 0)
    one = kv8.Cache(fmt, block, 2, 3, 8, 160)
    one.store(x, [0, 0])
    for a, b in ((0, 37), (37, 38), (38, 128), (128, 150)):
        many.store(x[:, a:b], [a, a])
    got = one.read()[..., :150, :].transpose(0, 3, 2, 1, 4)
    step = np.abs(x) / 16 if fmt == kv8.E4M3 else 0.5 * 2.0 ** -3      # max|x| < 16 = 2^-3 * 128
    assert np.all(np.abs(got - x) <= step + 2.0 ** -10)
    # 4 |first row|'s maximum is not always the block's: compare where scales agree
    same = one.scale == many.scale
    rep = np.repeat(same, block, axis=-1)[..., :160]
    assert np.mean(same) > 0.9
    assert np.array_equal(one.code[rep], many.code[rep])


def test_growth_rounds_again_and_restart_forgets():
    c = kv8.Cache(kv8.INT8, 16, 1, 1, 1, 32)
    put = lambda v, p: c.store(np.full((1, 1, 2, 1, 1), v), [p])  # noqa: E731
    put(3.0, 0)
    assert c.scale[0, 0, 0, 0] == 2.0 ** -5 and c.code[0, 0, 0, 0, 0] == 96
    put(1000.0, 1)
    assert c.scale[0, 0, 0, 0] == 8.0 and list(c.read()[0, 0, 0, :2, 0]) == [0.0, 1000.0]   # 3/8 rounds to 0
    put(math.inf, 2)
    assert math.isnan(c.scale[0, 0, 0, 0])
    put(1.0, 3)
    assert math.isnan(c.scale[0, 0, 0, 0])
    put(1.0, 0)
    assert c.scale[0, 0, 0, 0] == 2.0 ** -6 and c.read()[0, 0, 0, 0, 0] == 1.0


@pytest.mark.parametrize("fmt", [kv8.E4M3, kv8.INT8])
def test_pack_round_trip(fmt):
    rng = np.random.default_rng(2)
    c = kv8.Cache(fmt, 32, 2, 3, 64, 41)
    c.store(rng.standard_normal((2, 41, 2, 3, 64)), [0, 0])
    raw = c.pack(fill=9)
    assert raw.size == 2 * 3 * 2 * 48 * 64
    assert np.array_equal(kv8.unpack(raw, 2, 3, 64, 41), kv8.to_bytes(fmt, c.code))
    # the layout by its words: value of position 35, dimension 7, head 2 of sequence 1
    at = ((1 * 3 + 2) * 2 + 1) * 48 * 64 + (35 // 16) * 64 * 16 + 7 * 16 + 35 % 16
    assert raw[at] == kv8.to_bytes(fmt, c.code[1, 2, 1, 35, 7])
    at = ((1 * 3 + 2) * 2 + 0) * 48 * 64 + 35 * 64 + 7
    assert raw[at] == kv8.to_bytes(fmt, c.code[1, 2, 0, 35, 7])


@pytest.mark.parametrize("alibi", [0, 1])
def test_attention_is_torchs(alibi):
    rng = np.random.default_rng(3)
    B, n, H, KV, dh, S = 3, 2, 6, 2, 16, 40
    v = rng.standard_normal((B, KV, 2, S, dh))
    q = rng.standard_normal((B, n, H, dh))
    pos = [0, 38, None]
    o, a, _ = kv8.attention(v, q, pos, alibi)
    for b in (0, 1):
        c = pos[b] + n
        k, w = (torch.from_numpy(v[b, :, i, :c]).repeat_interleave(H // KV, 0) for i in (0, 1))
        qp, kp = torch.arange(pos[b], c)[:, None], torch.arange(c)[None]
        mask = torch.where(kp <= qp, 0.0, -math.inf).double()[None]
        if alibi:
            mask = mask - torch.tensor(kv8.slopes(H)).double()[:, None, None] * (qp - kp).clamp(min=0)
        want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q[b]).transpose(0, 1), k, w,
                                                                attn_mask=mask.expand(H, -1, -1))
        np.testing.assert_allclose(o[b], want.transpose(0, 1).numpy(), rtol=1e-12, atol=1e-12)
    assert not np.any(o[2]) and np.all(np.abs(o) <= a + 1e-12)
