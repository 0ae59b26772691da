"""A stack's caches cut and decoded over: prefill, steps that sum weights, eviction of
every layer, steps at the place behind what stayed."""
import dataclasses

import numpy as np
import pytest
import torch

import ld_inputs as inp
import paper_2609_05275_amd as ld
from oracle import kv4, w4
from tests.gpu_util import DEV, f64, rel, tol
from tests.test_gpu_kv4_stack import IDS, SHAPES, _adopt, _caches, _in_4_bits, _oracle_step, _prefill, _weights
from tests.test_gpu_layer import _buf, _cfg

pytestmark = pytest.mark.gpu


def _cut(kv, length, keep, recent, s_max):
    """The layers' caches cut to `keep` of `length` positions, which they are, and the cut
    caches' oracles."""
    out, refs, kept = [], [], []
    for k in kv:
        shape = (k.n_seq, k.n_kv_heads, k.d_head)
        probe = ld.kv4(None, None, *shape, s_max)
        to = ld.kv4(torch.full((ld.ld_kv4_code_bytes(probe),), 0xFF, dtype=torch.uint8, device=DEV),
                    torch.full((ld.ld_kv4_scale_bytes(probe),), 0xFF, dtype=torch.uint8, device=DEV), *shape, s_max,
                    sums=torch.full((*shape[:2], s_max), 1e9, device=DEV))
        idx = torch.full((*shape[:2], keep), -7, dtype=torch.int32, device=DEV)
        ld.ld_kv4_evict(k, to, length, keep, recent, idx, _buf(max(16, ld.ld_kv4_evict_ws_bytes(k, length, keep))))
        idx, sums = idx.cpu().numpy(), f64(k.tensors[2])
        code = kv4.from_codes(kv4.unpack(k.tensors[0].cpu().numpy(), *shape, k.s_max))
        scale = k.tensors[1].cpu().numpy().reshape(*shape[:2], 2, -1, k.d_head // 32)
        ref = kv4.Cache(*shape, s_max)
        for b in range(k.n_seq):
            for h in range(k.n_kv_heads):
                assert idx[b, h].tolist() == kv4.evict(sums[b, h], length, keep, recent), (b, h)
                ref.code[b, h, :, :keep] = code[b, h][:, idx[b, h]]
                ref.scale[b, h, :, :keep] = scale[b, h][:, idx[b, h]]
                ref.sums[b, h, :keep] = sums[b, h, idx[b, h]]
        assert np.array_equal(f64(to.tensors[2])[..., :keep], ref.sums[..., :keep])
        out.append(to)
        refs.append(ref)
        kept.append(idx)
    return out, refs, kept


@pytest.mark.parametrize("sh", SHAPES, ids=IDS)
@pytest.mark.parametrize("four", [False, True], ids=["bf16", "w4"])
def test_decoding_goes_on_after_an_eviction(sh, four):
    """Steps over what stayed against the oracle over the same codes (ALiBi: distances by
    place), the sums going on, and a second eviction by them."""
    sh = dataclasses.replace(sh, batch=3, seq=64)
    L, W = sh.n_layers, _weights(sh)
    if four:
        V = _in_4_bits(sh, W, [(w4.E2M1, 32), (w4.INT4, 32), (w4.INT4, 64), (w4.INT4, 128)])
        W = [({k: torch.from_numpy(np.asarray(v)).to(torch.bfloat16).to(DEV) for k, v in v64.items()}, v64) for _, v64 in V]
        wd, w64, step = [v[0] for v in V], [v[1] for v in V], ld.ld_stack_decode_w4
    else:
        wd, w64, step = [w[0] for w in W], [w[1] for w in W], ld.ld_stack_decode_kv4
    cfg, act = _cfg(sh), [1] * L
    X = inp.hidden(dataclasses.replace(sh, seq=128))
    kv = _caches(sh, 100, sums=True)
    _prefill(sh, W, kv, X[:, :64].contiguous())
    ws = _buf(ld.ld_decode_kv4_ws_bytes(cfg, 8, 100, sums=True))
    at = 64
    for n in (1, 6, 2):
        step(cfg, wd, X[:, at:at + n].contiguous().to(DEV), kv, at, n, ws)
        at += n
    for k in kv:      # each new row put a weight of 1 on a head's positions
        np.testing.assert_allclose(f64(k.tensors[2])[..., :at].sum(-1), at - 64, rtol=1e-4)
    for keep, recent, s_max in ((24, 6, 60), (13, 13, 40)):
        kv, refs, _ = _cut(kv, at, keep, recent, s_max)
        at = keep
        for i, n in enumerate((1, 5)):
            x = X[:, 90 + 6 * i:90 + 6 * i + n].contiguous()
            xd = x.to(DEV)
            step(cfg, wd, xd, kv, at, n, ws)
            want = _oracle_step(inp.f64(x), w64, refs, [at] * sh.batch, sh.n_heads, sh.kind, act)
            assert rel(f64(xd), want) < 1.5 * tol("bf16"), (keep, n)
            for l in range(L):
                _adopt(kv[l], refs[l], at, n)
                # (a weight's relative error is its score's, of bf16 queries and keys)
                assert rel(f64(kv[l].tensors[2][..., :at + n]), refs[l].sums[..., :at + n]) < 0.05
            at += n


def test_a_prompt_has_no_sums_of_its_own():
    """Right after a prefill every sum is zero, and of equal sums the first positions
    stay."""
    sh = dataclasses.replace(SHAPES[0], batch=2, seq=64)
    W = _weights(sh)
    kv = _caches(sh, 70, sums=True)
    _prefill(sh, W, kv, inp.hidden(sh))
    _, refs, kept = _cut(kv, 64, 20, 4, 20)
    for idx, ref in zip(kept, refs):
        assert (idx == np.r_[0:16, 60:64]).all() and not ref.sums[..., :20].any()
