"""Scores of the 4-bit attention where large and small products stand side by side:
float32 sums, nothing of the small ones lost."""
import numpy as np
import pytest
import torch

from tests.test_gpu_kv4 import DHS, Dev, check, rows

pytestmark = pytest.mark.gpu


def uneven(dh, small, keys, seed, each, sums=True):
    """Queries of +-1 in one of `each` dimensions and of `small` in the others, over random
    keys."""
    rng = np.random.default_rng(seed)
    dev = Dev(2, 2, dh, keys + 3, sums=sums)
    x = rows(rng, 2, keys, 2, 2, dh)
    dev.ref.store(x.double().numpy(), [0, 0])
    dev.upload([keys, keys])
    q = rng.uniform(0.5, 1.0, (2, 3, 4, dh)) * rng.choice([-1.0, 1.0], (2, 3, 4, dh)) * small
    q[..., ::each] = rng.choice([-1.0, 1.0], q[..., ::each].shape)
    return dev, torch.from_numpy(q).to(torch.bfloat16)


@DHS
@pytest.mark.parametrize("each", [8, 32])
@pytest.mark.parametrize("small", [2.0 ** -6, 2.0 ** -9, 2.0 ** -12, 2.0 ** -16])
def test_small_products_beside_large(dh, each, small):
    """The sums of weights, float32, within the bound of float32 scores (a matrix
    instruction that adds 8 products to 13 bits below their largest would be off by up to
    2^-14 of it a product: 3 to 30 times the bound)."""
    dev, q = uneven(dh, small, 20, 1, each)
    check(dev, q, [17, 17])


@DHS
def test_large_products_that_cancel(dh):
    """Two dimensions 2^8 times the others whose products cancel in every key: what is left
    is the others' sum."""
    rng = np.random.default_rng(2)
    dev = Dev(1, 2, dh, 60, sums=True)
    x = rows(rng, 1, 60, 2, 2, dh)
    x[:, :, 0, :, 9] = x[:, :, 0, :, 8]
    x[:, :, 0, :, dh - 1] = x[:, :, 0, :, dh - 2]
    dev.ref.store(x.double().numpy(), [0])
    dev.upload()
    q = rows(rng, 1, 2, 4, dh)
    for i in (8, dh - 2):
        q[..., i] = 256.0
        q[..., i + 1] = -256.0
    check(dev, q, [58])
