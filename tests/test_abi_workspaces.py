"""A scratch buffer made for a step of so many rows also holds every step of
fewer (no GPU: the sizes are the host's)."""
import pytest

import paper_2609_05275_amd as ld
from tests.test_abi_kv8 import desc


def grows(sizes):
    assert sizes[0] > 0
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("s_max", [1, 300, 5000, 131072, 1 << 20])
@pytest.mark.parametrize("n_seq,kv_heads,heads", [(1, 1, 1), (1, 8, 64), (2, 8, 32), (1, 1, 12), (1, 4, 20), (3, 2, 34),
                                                  (40, 8, 64)])
def test_attention_of_fewer_rows(n_seq, kv_heads, heads, s_max):
    kv = desc(n_seq=n_seq, n_kv_heads=kv_heads, s_max=s_max)
    grows([ld.ld_attn_decode_kv8_ws_bytes(kv, heads, n) for n in range(1, 9)])


@pytest.mark.parametrize("batch", [1, 2, 9, 17, 33, 64])        # 64 rows are passed at different n_new
@pytest.mark.parametrize("d,heads,f", [(512, 8, 1408), (1024, 16, 2816), (2560, 20, 6912), (4096, 32, 11008)])
def test_decoding_steps_of_fewer_rows(batch, d, heads, f):
    cfg = ld.config(batch, 128, d, heads, f)
    for s_max in (64, 2048, 100000):
        grows([ld.ld_decode_ws_bytes(cfg, n, s_max) for n in range(1, 9)])
        grows([ld.ld_decode_kv8_ws_bytes(cfg, n, s_max) for n in range(1, 9)])
