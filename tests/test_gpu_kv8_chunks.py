"""The 8-bit cache's attention over several chunks of a host-known length: with
several row tiles, with the same bits again, and within scratch made once for
the widest step."""
import dataclasses

import pytest
import torch

import ld_inputs as inp
import paper_2609_05275_amd as ld
from oracle import kv8
from tests.gpu_util import DEV
from tests.test_gpu_kv8 import DHS, FMTS, check, filled, rows
from tests.test_gpu_kv8_prof import profiled
from tests.test_gpu_kv8_stack import _caches, _prefill, _weights
from tests.test_gpu_layer import SMALL_BF16_128, _cfg

pytestmark = pytest.mark.gpu


@FMTS
@DHS
@pytest.mark.parametrize("n_seq,kvh,group,n", [(1, 1, 3, 7), (1, 3, 5, 8), (2, 2, 8, 8), (1, 5, 17, 2), (3, 4, 24, 4)])
@pytest.mark.parametrize("keys", [2500, 4001])
def test_row_tiles_over_chunks(fmt, dh, n_seq, kvh, group, n, keys):
    """Two to six row tiles, the last one part empty; units of (head, chunk) that
    are no multiple of the eight of a set."""
    dev, rng = filled(fmt, 64, n_seq, kvh, dh, keys, group)
    q = rows(rng, n_seq, n, kvh * group, dh)
    merges = profiled("ld_attn_decode_kv8_combine", lambda: check(dev, q, [keys - n] * n_seq, alibi=n % 2))
    assert merges["launches"] == 2


@FMTS
@pytest.mark.parametrize("group,n", [(1, 1), (6, 5)])
def test_the_same_bits_again(fmt, group, n):
    """NaN scales and queries among them, over scratch that holds anything."""
    keys, H = 2900, 2 * group
    dev, rng = filled(fmt, 16, 2, 2, 128, keys, n)
    dev.scales.view(2, 2, 2, -1)[0, 1, 0, 20] = float("nan")
    dev.scales.view(2, 2, 2, -1)[1, 0, 1, 150] = float("nan")
    qkv = torch.zeros(2 * n, (H + 4) * 128, dtype=torch.bfloat16)
    qkv[:, :H * 128] = rows(rng, 2 * n, H * 128)
    qkv[0, 3] = float("inf")
    qkv = qkv.to(DEV)
    ws = torch.empty(ld.ld_attn_decode_kv8_ws_bytes(dev.kv, H, n), dtype=torch.uint8, device=DEV)
    seen = []
    for fill in (0, 0xFF, 0x7F, 0x11):
        ws.fill_(fill)
        o = torch.full((2 * n, H * 128), float(fill), dtype=torch.bfloat16, device=DEV)
        ld.ld_attn_decode_kv8(dev.kv, H, keys - n, n, qkv, o, ws)
        seen.append(o.view(torch.int16).clone())
    for s in seen[1:]:
        assert torch.equal(s, seen[0])
    nan = torch.isnan(seen[0].view(torch.bfloat16)).view(2, n, 2, group * 128).all(-1)
    assert bool(nan[0, :, 1].all()) and bool(nan[1, :, 0].all()) and not bool(nan[1, :, 1].any())


@pytest.mark.parametrize("n_seq,kvh,H", [(1, 2, 16), (2, 1, 9)])
def test_scratch_of_the_widest_step(n_seq, kvh, H):
    """What the query asks for at eight rows holds steps of eight to one, and
    nothing behind it is written."""
    keys = 6000
    dev, rng = filled(kv8.E4M3, 128, n_seq, kvh, 64, keys, H)
    size = ld.ld_attn_decode_kv8_ws_bytes(dev.kv, H, 8)
    ws = torch.full((size + 4096,), 77, dtype=torch.uint8, device=DEV)
    for seq_pos in (None, torch.full((n_seq,), keys - 8, dtype=torch.int32, device=DEV)):
        for n in range(8, 0, -1):
            qkv = rows(rng, n_seq * n, (H + 2 * kvh) * 64).to(DEV)
            o, alone = (torch.zeros(n_seq * n, H * 64, dtype=torch.bfloat16, device=DEV) for _ in range(2))
            ld.ld_attn_decode_kv8(dev.kv, H, keys - 8, n, qkv, o, ws[:size], seq_pos=seq_pos)
            own = torch.empty(ld.ld_attn_decode_kv8_ws_bytes(dev.kv, H, n), dtype=torch.uint8, device=DEV)
            ld.ld_attn_decode_kv8(dev.kv, H, keys - 8, n, qkv, alone, own, seq_pos=seq_pos)
            assert torch.equal(o, alone)
    assert bool((ws[size:] == 77).all())


def test_stack_scratch_of_the_widest_step():
    """Decoding steps of eight rows to one of nine sequences in one buffer: up to 64
    rows in all use split-K sums, 72 do not."""
    sh = dataclasses.replace(SMALL_BF16_128, batch=9, seq=64)
    cfg, W = _cfg(sh), _weights(sh)
    kv = _caches(sh, kv8.INT8, 32, 100)
    _prefill(sh, W, kv, inp.hidden(sh))
    bf = [torch.zeros(9, 100, 2 * sh.d_model, dtype=torch.bfloat16, device=DEV) for _ in range(sh.n_layers)]
    size8, size16 = ld.ld_decode_kv8_ws_bytes(cfg, 8, 100), ld.ld_decode_ws_bytes(cfg, 8, 100)
    ws8, ws16 = (torch.full((s + 4096,), 77, dtype=torch.uint8, device=DEV) for s in (size8, size16))
    for n in range(8, 0, -1):
        x = inp.hidden(dataclasses.replace(sh, seq=n)).to(DEV)
        y = x.clone()
        ld.ld_stack_decode_kv8(cfg, [w[0] for w in W], x, kv, 64, n, ws8[:size8])
        ld.ld_stack_decode(cfg, [w[0] for w in W], y, bf, 100, 64, n, ws16[:size16])
        assert bool(torch.isfinite(x).all()) and bool(torch.isfinite(y).all())
    assert bool((ws8[size8:] == 77).all()) and bool((ws16[size16:] == 77).all())
