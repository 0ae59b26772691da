"""Attention over the 4-bit cache by queries near the smallest numbers."""
import numpy as np
import pytest

from tests.test_gpu_kv4 import DHS, Dev, check, rows

pytestmark = pytest.mark.gpu


@DHS
@pytest.mark.parametrize("small", [2.0 ** -113, 2.0 ** -115, 2.0 ** -119, 2.0 ** -123])
def test_small_queries(dh, small):
    """Against keys as large: products around 1, subnormal queries (below 2^-126) among
    them."""
    rng = np.random.default_rng(8)
    dev = Dev(1, 2, dh, 120)
    x = rows(rng, 1, 120, 2, 2, dh)
    x[:, :, 0] *= 1.0 / small
    dev.ref.store(x.double().numpy(), [0])
    dev.upload()
    q = rows(rng, 1, 3, 4, dh) * small
    q[0, 0, 0, 1] = 2.0 ** -133
    check(dev, q, [117])


@DHS
@pytest.mark.parametrize("top", [2.0 ** -113, 2.0 ** -118, 2.0 ** -126])
def test_small_queries_beside_larger(dh, top):
    """One dimension of 32 at `top`, where the keys are zero, the others down to 2^-13 of it."""
    rng = np.random.default_rng(9)
    dev = Dev(1, 2, dh, 120)
    x = rows(rng, 1, 120, 2, 2, dh)
    x[:, :, 0] *= 2.0 ** 123
    x[:, :, 0, :, 7::32] = 0.0
    dev.ref.store(x.double().numpy(), [0])
    dev.upload()
    q = rows(rng, 1, 3, 4, dh) * max(2.0 ** -126, top * 2.0 ** -13)
    q[..., 7::32] = top
    check(dev, q, [117])
