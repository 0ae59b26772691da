"""What the profiling hook says of the 8-bit cache's launches."""
import pytest
import torch

import paper_2609_05275_amd as ld
from oracle import kv8
from tests.gpu_util import DEV
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
    computed where the host knows the lengths, and 0 where it does not."""
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
    for kernel in ("ld_attn_decode_kv8_k", "ld_attn_decode_kv8_combine"):
        r = profiled(kernel, lambda: attend(dev, q, [keys - 1, None], seq_pos=True))
        assert r["launches"] == 2 and r["ms"] > 0 and r["flops"] == r["bytes"] == 0


def test_store_and_load():
    dev, rng = filled(kv8.INT8, 32, 3, 2, 64, 100, 2)
    n = 3 * 5 * 2 * 64 * 2          # values of five rows
    x = rows(rng, 3, 5, 2, 2, 64)
    r = profiled("ld_kv8_store_k", lambda: dev.store(x, [95] * 3))
    assert r["launches"] == 1 and r["bytes"] == 3.0 * n
    r = profiled("ld_kv8_store_k", lambda: dev.store(x, [95, None, 7], seq_pos=True))
    assert r["launches"] == 1 and r["bytes"] == 0
    out = torch.zeros(3, 5, 4 * 64, dtype=torch.bfloat16, device=DEV)
    r = profiled("ld_kv8_load_k", lambda: ld.ld_kv8_load(dev.kv, 90, 5, out))
    assert r["launches"] == 1 and r["bytes"] == 3.0 * n
    ends = torch.tensor([95, 0, 7], dtype=torch.int32, device=DEV)
    r = profiled("ld_kv8_load_k", lambda: ld.ld_kv8_load(dev.kv, 90, 5, out, seq_len=ends))
    assert r["launches"] == 1 and r["bytes"] == 0
