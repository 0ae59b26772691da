"""Eviction from the 4-bit cache by its positions' sums against the oracle: which
positions stay, and their bits, exactly."""
import math

import numpy as np
import pytest
import torch

import paper_2609_05275_amd as ld
from oracle import kv4
from tests.gpu_util import DEV, f64
from tests.test_gpu_kv4 import DHS, FILL, Dev, check, filled, rows

pytestmark = pytest.mark.gpu


def evict(dev, to, length, keep, recent, seq_len=None):
    n, kvh = dev.shape[:2]
    idx = torch.full((n, kvh, keep), -7, dtype=torch.int32, device=DEV)
    ws = torch.empty(ld.ld_kv4_evict_ws_bytes(dev.kv, length, keep), dtype=torch.uint8, device=DEV)
    ws.fill_(0xEE)
    sl = None if seq_len is None else torch.tensor(seq_len, dtype=torch.int32, device=DEV)
    before = [t.clone() for t in (dev.codes, dev.scales, dev.sums)]
    ld.ld_kv4_evict(dev.kv, to.kv, length, keep, recent, idx, ws, seq_len=sl)
    for a, b in zip(before, (dev.codes, dev.scales, dev.sums)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    return idx.cpu().numpy()


def compare(dev, to, idx, lens, keep, recent):
    n, kvh = dev.shape[:2]
    code, scale = dev.raw()
    tc, ts = to.raw()
    sums, tsums = f64(dev.sums), None if to.sums is None else f64(to.sums)
    for b in range(n):
        for h in range(kvh):
            want = kv4.evict(sums[b, h], lens[b], keep, recent)
            k = len(want)
            assert idx[b, h, :k].tolist() == want and (idx[b, h, k:] == -1).all(), (b, h)
            np.testing.assert_array_equal(tc[b, h, :, :k], code[b, h][:, want])
            np.testing.assert_array_equal(ts[b, h, :, :k], scale[b, h][:, want])
            assert np.all(tc[b, h, :, k:] == 15) and np.all(ts[b, h, :, k:] == FILL)
            if tsums is not None:
                np.testing.assert_array_equal(tsums[b, h, :k], sums[b, h, want])
                assert np.all(tsums[b, h, k:] == 1e9)


def weights(rng, *shape):
    """Few large, many small, some zero."""
    x = np.exp(3 * rng.standard_normal(shape)).astype(np.float32)
    return torch.from_numpy(np.where(rng.random(shape) < 0.2, 0.0, x).astype(np.float32))


@DHS
@pytest.mark.parametrize("length,keep,recent", [(1, 1, 0), (1, 5, 5), (9, 8, 8), (9, 8, 0), (300, 1, 0), (300, 1, 1),
                                                (300, 37, 8), (300, 299, 1), (300, 300, 0), (300, 310, 20),
                                                (5000, 700, 100), (5000, 700, 700)])
def test_lengths(dh, length, keep, recent):
    dev, rng = filled(2, 3, dh, length, length + keep, sums=True)
    dev.sums[:, :, :length] = weights(rng, 2, 3, length).to(DEV)
    to = Dev(2, 3, dh, keep + 3, sums=True)
    compare(dev, to, evict(dev, to, length, keep, recent), [length] * 2, keep, recent)


@DHS
def test_ragged(dh):
    """Each sequence its own length, from none to all; outside [0, len]: none."""
    dev, rng = filled(7, 2, dh, 2100, 1, sums=True)
    dev.sums[:, :, :2100] = weights(rng, 7, 2, 2100).to(DEV)
    lens = [0, 1, 63, 64, 65, 2100, 1025]
    for keep, recent in ((64, 16), (1000, 0)):
        to = Dev(7, 2, dh, keep, sums=True)
        compare(dev, to, evict(dev, to, 2100, keep, recent, seq_len=lens), lens, keep, recent)
    to = Dev(7, 2, dh, 64, sums=True)
    got = evict(dev, to, 1000, 64, 4, seq_len=[-1, 1001, 10 ** 9, 1000, 999, -2 ** 31, 2 ** 31 - 1])
    compare(dev, to, got, [0, 0, 0, 1000, 999, 0, 0], 64, 4)


KINDS = ["equal", "zeros", "two", "nan", "negative", "close", "huge"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("length,keep,recent", [(2500, 600, 50), (700, 699, 0), (130, 64, 63)])
def test_ties_and_odd_values(kind, length, keep, recent):
    dev, rng = filled(2, 2, 64, length, 3, sums=True)
    s = {"equal": np.full((2, 2, length), 0.3), "zeros": np.where(rng.random((2, 2, length)) < 0.5, 0.0, -0.0),
         "two": rng.integers(0, 2, (2, 2, length)), "nan": rng.random((2, 2, length)),
         "negative": rng.standard_normal((2, 2, length)), "close": 1 + rng.integers(0, 300, (2, 2, length)) * 2.0 ** -23,
         "huge": rng.standard_normal((2, 2, length)) * 1e38}[kind].astype(np.float32)
    if kind == "nan":
        s[rng.random(s.shape) < 0.1] = math.nan
        s[rng.random(s.shape) < 0.1] = math.inf
    if kind == "huge":
        s[rng.random(s.shape) < 0.3] = -math.inf
        s[rng.random(s.shape) < 0.1] = 1e-40
    dev.sums[:, :, :length] = torch.from_numpy(s).to(DEV)
    to = Dev(2, 2, 64, keep, sums=True)
    compare(dev, to, evict(dev, to, length, keep, recent), [length] * 2, keep, recent)


@pytest.mark.parametrize("n_seq,kvh,length,keep,recent", [(1, 1, 131072, 16384, 1024), (1, 2, 70001, 33333, 0),
                                                          (40, 8, 1500, 300, 30), (1, 1, 20000, 19999, 10000)])
def test_long_and_many(n_seq, kvh, length, keep, recent):
    """Many pieces a head, many heads; without sums in the smaller cache."""
    rng = np.random.default_rng(length)
    dev = Dev(n_seq, kvh, 64, length, sums=True)
    dev.codes.copy_(torch.from_numpy(rng.integers(0, 256, dev.codes.numel(), dtype=np.uint8)))
    dev.scales.copy_(torch.from_numpy(rng.integers(27, 253, dev.scales.numel(), dtype=np.uint8)))
    dev.sums.copy_(weights(rng, n_seq, kvh, length))
    to = Dev(n_seq, kvh, 64, keep)
    compare(dev, to, evict(dev, to, length, keep, recent), [length] * n_seq, keep, recent)


@DHS
def test_decoding_goes_on_over_what_stayed(dh):
    """Prompt, steps that sum weights, eviction, and steps over the smaller cache."""
    rng = np.random.default_rng(dh)
    B, kvh, H, n0 = 2, 2, 4, 500
    dev = Dev(B, kvh, dh, 520, sums=True)
    dev.store(rows(rng, B, n0, 2, kvh, dh), [0, 0], n_heads=H)
    ws = torch.empty(ld.ld_attn_decode_kv4_ws_bytes(dev.kv, H, 4), dtype=torch.uint8, device=DEV)
    at = n0
    for n in (1, 4, 1):
        dev.store(rows(rng, B, n, 2, kvh, dh), [at] * B, n_heads=H)
        ld.ld_attn_decode_kv4(dev.kv, H, at, n, rows(rng, B * n, (H + 2 * kvh) * dh).to(DEV),
                              torch.zeros(B * n, H * dh, dtype=torch.bfloat16, device=DEV), ws)
        at += n
    # each step's rows put a weight of 1 a query head on a head's positions
    np.testing.assert_allclose(f64(dev.sums[:, :, :at]).sum(-1), (1 + 4 + 1) * H // kvh, rtol=1e-4)
    to = Dev(B, kvh, dh, 200, sums=True)
    idx = evict(dev, to, at, 120, 16)
    compare(dev, to, idx, [at] * B, 120, 16)
    for b in range(B):
        for h in range(kvh):
            to.ref.code[b, h, :, :120] = dev.ref.code[b, h][:, idx[b, h]]
            to.ref.scale[b, h, :, :120] = dev.ref.scale[b, h][:, idx[b, h]]
    at = 120
    for n in (1, 3):
        to.store(rows(rng, B, n, 2, kvh, dh), [at] * B, n_heads=H)
        check(to, rows(rng, B, n, H, dh), [at] * B)
        at += n


def test_captured_and_replayed():
    """A captured eviction follows the sums and lengths that it finds, on each replay."""
    dev, rng = filled(3, 2, 64, 1500, 9, sums=True)
    keep, recent = 200, 32
    to, to2 = Dev(3, 2, 64, keep, sums=True), Dev(3, 2, 64, keep, sums=True)
    idx, idx2 = (torch.zeros(3, 2, keep, dtype=torch.int32, device=DEV) for _ in range(2))
    sl = torch.tensor([1500, 900, 100], dtype=torch.int32, device=DEV)
    ws, ws2 = (torch.empty(ld.ld_kv4_evict_ws_bytes(dev.kv, 1500, keep), dtype=torch.uint8, device=DEV) for _ in range(2))
    call = lambda t, i, w: ld.ld_kv4_evict(dev.kv, t.kv, 1500, keep, recent, i, w, seq_len=sl)  # noqa: E731
    call(to, idx, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(to, idx, ws)
    for i in range(4):
        dev.sums[:, :, :1500] = weights(rng, 3, 2, 1500).to(DEV)
        sl.copy_(torch.tensor([1500 - 300 * i, 900 + i, 199 + i], dtype=torch.int32))
        call(to2, idx2, ws2)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(idx, idx2)
        compare(dev, to2, idx2.cpu().numpy(), sl.tolist(), keep, recent)
        for b, n in enumerate(sl.tolist()):
            k = min(n, keep)
            assert torch.equal(to.sums[b, :, :k], to2.sums[b, :, :k])
        to2 = Dev(3, 2, 64, keep, sums=True)
