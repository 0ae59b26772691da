"""Eviction of heads that go in pieces (more than 8192 positions): lengths on the
device, ties and odd values across pieces, everything recent, replays over scratch
that an earlier call left."""
import math

import numpy as np
import pytest
import torch

import paper_2609_05275_amd as ld
from tests.gpu_util import DEV
from tests.test_gpu_kv4 import Dev
from tests.test_gpu_kv4_evict import KINDS, compare, evict, weights

pytestmark = pytest.mark.gpu


def long_cache(n_seq, kvh, length, seed):
    """Random codes and scales, sums of few large, many small and some zero weights."""
    rng = np.random.default_rng(seed)
    dev = Dev(n_seq, kvh, 64, length, sums=True)
    dev.codes.copy_(torch.from_numpy(rng.integers(0, 256, dev.codes.numel(), dtype=np.uint8)))
    dev.scales.copy_(torch.from_numpy(rng.integers(27, 253, dev.scales.numel(), dtype=np.uint8)))
    dev.sums.copy_(weights(rng, n_seq, kvh, length))
    return dev, rng


LENS = [0, 1, 300, 301, 4095, 4096, 4097, 8192, 8193, 12288, 12289, 20000]


@pytest.mark.parametrize("keep,recent", [(300, 0), (300, 300), (300, 37), (4097, 1), (12000, 9000)])
def test_ragged(keep, recent):
    """From none to all, at both sides of a piece's end; some shorter than what is kept."""
    dev, _ = long_cache(len(LENS), 1, 20000, keep + recent)
    to = Dev(len(LENS), 1, 64, keep, sums=True)
    compare(dev, to, evict(dev, to, 20000, keep, recent, seq_len=LENS), LENS, keep, recent)


def test_lengths_outside():
    dev, _ = long_cache(6, 2, 9000, 1)
    to = Dev(6, 2, 64, 200, sums=True)
    got = evict(dev, to, 8500, 200, 10, seq_len=[-1, 8501, 8500, 2 ** 31 - 1, -2 ** 31, 8499])
    compare(dev, to, got, [0, 0, 8500, 0, 0, 8499], 200, 10)


@pytest.mark.parametrize("length,keep,recent", [(8193, 1, 0), (8193, 1, 1), (8193, 8192, 0), (8193, 8193, 5), (8193, 9000, 0),
                                                (16385, 4096, 4096), (12289, 12288, 4096)])
def test_lengths(length, keep, recent):
    dev, _ = long_cache(1, 2, length, length + keep)
    to = Dev(1, 2, 64, keep + 3, sums=True)
    compare(dev, to, evict(dev, to, length, keep, recent), [length], keep, recent)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("length,keep,recent", [(9000, 5000, 100), (12290, 12289, 0), (20000, 300, 299)])
def test_ties_and_odd_values(kind, length, keep, recent):
    dev, rng = long_cache(1, 2, length, 3)
    shape = (1, 2, length)
    s = {"equal": np.full(shape, 0.3), "zeros": np.where(rng.random(shape) < 0.5, 0.0, -0.0),
         "two": rng.integers(0, 2, shape), "nan": rng.random(shape), "negative": rng.standard_normal(shape),
         "close": 1 + rng.integers(0, 300, shape) * 2.0 ** -23,
         "huge": rng.standard_normal(shape) * 1e38}[kind].astype(np.float32)
    if kind == "nan":
        s[rng.random(s.shape) < 0.1] = math.nan
        s[rng.random(s.shape) < 0.1] = math.inf
    if kind == "huge":
        s[rng.random(s.shape) < 0.3] = -math.inf
        s[rng.random(s.shape) < 0.1] = 1e-40
    dev.sums.copy_(torch.from_numpy(s))
    to = Dev(1, 2, 64, keep, sums=True)
    compare(dev, to, evict(dev, to, length, keep, recent), [length], keep, recent)


def test_captured_and_replayed():
    """Two captured calls share scratch, which each finds as the other left it; sums and
    lengths change between the replays."""
    devs = [long_cache(3, 2, n, n) for n in (9000, 17000)]
    keep, recent = 700, 32
    size = max(ld.ld_kv4_evict_ws_bytes(dev.kv, dev.shape[3], keep) for dev, _ in devs)
    ws = torch.full((size,), 0xEE, dtype=torch.uint8, device=DEV)
    sls = [torch.tensor([dev.shape[3], 5000, 100], dtype=torch.int32, device=DEV) for dev, _ in devs]
    idxs = [torch.zeros(3, 2, keep, dtype=torch.int32, device=DEV) for _ in devs]
    tos = [Dev(3, 2, 64, keep, sums=True) for _ in devs]

    def call(i):
        dev, to = devs[i][0], tos[i]
        ld.ld_kv4_evict(dev.kv, to.kv, dev.shape[3], keep, recent, idxs[i], ws, seq_len=sls[i])

    graphs = []
    for i in range(2):
        call(i)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(i)
    for turn in range(4):
        for i in range(2) if turn % 2 else (1, 0):
            dev, rng = devs[i]
            n = dev.shape[3]
            dev.sums.copy_(weights(rng, 3, 2, n))
            lens = [n - 3000 * turn, 4096 + turn, 699 + turn]
            sls[i].copy_(torch.tensor(lens, dtype=torch.int32))
            for t in (tos[i].codes, tos[i].scales):
                t.fill_(0xFF)
            tos[i].sums.fill_(1e9)
            graphs[i].replay()
            torch.cuda.synchronize()
            compare(dev, tos[i], idxs[i].cpu().numpy(), [k if 0 <= k <= n else 0 for k in lens], keep, recent)
