"""What the profiling hook says of the 8-bit cache's launches."""
import pytest
import torch

import paper_2609_05275_amd as ld
from oracle import kv8
from tests.test_gpu_kv8 import attend, filled, rows

pytestmark = pytest.mark.gpu


def profiled(kernel, call):
    ld.ld_prof_start(kernel)
    try:
        call()
        torch.cuda.synchronize()
        return ld.ld_prof_result()
    finally:
        ld.ld_prof_stop()


def test_attention():
    """Two calls of several chunks: the merge under its own name; what was read and
    computed."""
    keys, H, dh = 3000, 4, 128
    dev, rng = filled(kv8.E4M3, 64, 2, 2, dh, keys, 1)
    q = rows(rng, 2, 1, H, dh)
    r = profiled("ld_attn_decode_kv8_k", lambda: attend(dev, q, [keys - 1] * 2))
    assert r["launches"] == 2 and r["ms"] > 0
    assert r["flops"] == 2 * 4.0 * 2 * H * dh * keys
    assert r["bytes"] == 2 * (2.0 * 2 * 2 * dh * keys + 4 * 2 * H * dh)
    m = profiled("ld_attn_decode_kv8_combine", lambda: attend(dev, q, [keys - 1] * 2))
    assert m["launches"] == 2 and m["ms"] > 0 and m["bytes"] > 0
    short = profiled("ld_attn_decode_kv8_combine", lambda: attend(dev, q, [9] * 2))
    assert short["launches"] == 0
