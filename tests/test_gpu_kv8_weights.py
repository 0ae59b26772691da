"""How many bits of a softmax weight the 8-bit cache's attention keeps: values
that cancel, so that neither the output's rounding nor sums over many keys hide
the weights' errors."""
import math

import numpy as np
import pytest
import torch

from oracle import kv8
from tests.test_gpu_kv8 import DHS, FMTS, Dev, attend

pytestmark = pytest.mark.gpu

NK = 4      # keys whose values are not zero
U = 2.0 ** -24


def bf16(x):
    """float64 rounded to bf16's 8 bits, ties to even."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(m * 256.0), e - 8)


def two_parts(w):
    """What two bf16 parts leave of a weight, relative to it."""
    w = w.astype(np.float32).astype(np.float64)
    return (w - bf16(w) - bf16(w - bf16(w))) / w


def cancelling(fmt, dh, seed):
    """Queries, keys and values of NK positions: scores q_i k_i / sqrt(dh) in (-0.6,
    0), one product each, so that they are exact but for their factors; of those
    some that two bf16 parts hold badly, half of them too large and half too small (errors of
    one sign would scale a sum that cancels), a few steps of float32 either way; values (NK x dh, of the format, one
    scale) whose weighted sums are 2^-12 of their magnitudes and less."""
    rng = np.random.default_rng(seed)
    code = rng.integers(8, 16, 4096) * 2.0 ** rng.integers(-1, 3, 4096)       # 4 bits: both formats have them
    q = bf16(rng.uniform(0.01, 0.1, 4096) * math.sqrt(dh / 64.0))
    s = -q * code / math.sqrt(dh)
    s, first = np.unique(s, return_index=True)
    q, code = q[first], code[first]
    near = np.stack([two_parts(np.exp(s) + n * U) for n in range(-4, 5)])
    low, high = near.min(0), near.max(0)
    ok = s > -0.6
    i = np.concatenate((np.argsort(-np.where(ok, low, -1.0))[:NK // 2], np.argsort(np.where(ok, high, 1.0))[:NK // 2]))
    w = np.exp(s[i])
    v = np.empty((NK, dh))
    for d in range(dh):
        many = (1 << 17, NK)
        c = rng.integers(8, 128, many) if fmt == kv8.INT8 else rng.integers(8, 16, many) * 2.0 ** rng.integers(0, 5, many)
        c = c * rng.choice([-1.0, 1.0], many)
        v[:, d] = c[np.argmin(np.abs(c @ w) / (np.abs(c) @ w))]
    return q[i], -code[i], w, v


def limit(fmt, dh, q, k, w, v):
    """Error of sum_i w_i v_i, in units of sum_i w_i |v_i|.  A base-2 score t = x f,
    |t| < 0.9: f's three roundings and the product's (u each), the maximum 0; the
    exponential 2 u; then the products' sum, at most three parts of NK terms, u each,
    and the waves' and chunks' sums, NK of which are not zero."""
    t = np.max(np.abs(np.log2(w)))
    return (math.log(2.0) * 4 * t + 2 + 4 * NK) * U


@FMTS
@DHS
@pytest.mark.parametrize("keys", [5, 40, 1500])
def test_attn_weights_in_24_bits(fmt, dh, keys):
    """In one wave; in one chunk; over chunks and their merge."""
    q, k, w, v = cancelling(fmt, dh, keys + dh)
    far = limit(fmt, dh, q, k, w, v)
    a, o = w @ np.abs(v), w @ v
    # the case can tell: two parts would leave more than twice the bound, rounded
    # outputs a small part of it
    assert np.max(np.abs((two_parts(w) * w) @ v) / a) > 2 * far
    assert np.max(np.abs(o) / a) * 2.0 ** -8 < far / 2
    rng = np.random.default_rng(keys)
    at = np.sort(rng.choice(keys - 1, NK, replace=False))       # the last position's key and value are zeros
    x = torch.zeros(1, keys, 2, 1, dh, dtype=torch.float64)
    for i, p in enumerate(at):
        x[0, p, 0, 0, i] = k[i]
        x[0, p, 1, 0] = torch.from_numpy(v[i])
    dev = Dev(fmt, 128, 1, 1, dh, keys)
    dev.ref.store(x.numpy(), [0])
    np.testing.assert_array_equal(np.nan_to_num(dev.ref.read())[0, 0, :, :keys].transpose(1, 0, 2), x[0, :, :, 0].numpy())
    dev.upload()
    query = torch.zeros(1, 1, 1, dh, dtype=torch.bfloat16)
    query[0, 0, 0, :NK] = torch.from_numpy(q).to(torch.bfloat16)
    got = attend(dev, query, [keys - 1])[0, 0, 0]
    total = np.sum(w) + keys - NK                                # the other scores are 0
    assert np.all(np.abs(got * total - o) <= 2.0 ** -8 * np.abs(o) + far * a + keys * U * np.abs(o))
