"""Prefill and decoding of a stack over 8-bit caches (ld_stack_eval_kv8,
ld_stack_decode_kv8) against the bf16 path and the float64 oracle."""
import dataclasses

import numpy as np
import pytest
import torch

import ld_inputs as inp
import paper_2609_05275_amd as ld
from oracle import block, kv8
from tests.gpu_util import DEV, f64, layer_weights_dev, rel, tol
from tests.test_gpu_layer import SMALL_BF16, SMALL_BF16_128, SMALL_P, SMALL_P_128, _buf, _cfg

pytestmark = pytest.mark.gpu

SHAPES = [SMALL_BF16, SMALL_P, SMALL_BF16_128, SMALL_P_128]
IDS = ["small", "paper_small", "small_dh128", "paper_small_dh128"]
FMTS = pytest.mark.parametrize("fmt", [kv8.E4M3, kv8.INT8], ids=["e4m3", "int8"])


def _caches(sh, fmt, blk, s_max):
    dh = sh.d_model // sh.n_heads
    code = ld.LD_KV8_E4M3 if fmt == kv8.E4M3 else ld.LD_KV8_INT8
    out = []
    for _ in range(sh.n_layers):
        probe = ld.kv8(None, None, code, blk, sh.batch, sh.n_heads, dh, s_max)
        codes = torch.full((ld.ld_kv8_code_bytes(probe),), 0x7F, dtype=torch.uint8, device=DEV)
        scales = torch.full((ld.ld_kv8_scale_bytes(probe) // 4,), float("nan"), device=DEV)
        out.append(ld.kv8(codes, scales, code, blk, sh.batch, sh.n_heads, dh, s_max))
    return out


def _copy(kv):
    return [ld.kv8(k.tensors[0].clone(), k.tensors[1].clone(), k.format, k.block, k.n_seq, k.n_kv_heads, k.d_head,
                   k.s_max) for k in kv]


def _weights(sh):
    return [layer_weights_dev(sh, l, gain_jitter=True) for l in range(sh.n_layers)]


def _prefill(sh, W, kv, x, active=None):
    xd = x.to(DEV)
    ld.ld_stack_eval_kv8(_cfg(sh), [w[0] for w in W], xd, _buf(ld.ld_eval_ws_bytes(_cfg(sh))), kv, active=active)
    return xd


def _split(kv, n_heads):
    """A bf16 cache [B, S, 2 d] as rows [B, S, 2, H, dh] in float64."""
    B, S, d2 = kv.shape
    return f64(kv).reshape(B, S, 2, n_heads, d2 // 2 // n_heads)


@pytest.mark.parametrize("sh", SHAPES, ids=IDS)
@FMTS
def test_prefill(sh, fmt):
    """Hidden states bit for bit ld_stack_eval's; caches the oracle's codes of
    the keys and values it stores; skipped layers' caches untouched."""
    L, S = sh.n_layers, sh.seq
    act = [1] * (L - 1) + [0]
    W, x = _weights(sh), inp.hidden(sh)
    cfg = _cfg(sh)
    want = x.to(DEV)
    bf = [torch.zeros(sh.batch, S, 2 * sh.d_model, dtype=torch.bfloat16, device=DEV) for _ in range(L)]
    ld.ld_stack_eval(cfg, [w[0] for w in W], want, _buf(ld.ld_eval_ws_bytes(cfg)), active=act, kv=bf, s_max=S)
    kv = _caches(sh, fmt, 32, S + 40)
    kv[-1] = None
    got = _prefill(sh, W, kv, x, active=act)
    assert torch.equal(got, want)
    dh = sh.d_model // sh.n_heads
    for l in range(L - 1):
        ref = kv8.Cache(fmt, 32, sh.batch, sh.n_heads, dh, S + 40)
        ref.store(_split(bf[l], sh.n_heads), [0] * sh.batch)
        raw = kv8.unpack(kv[l].tensors[0].cpu().numpy(), sh.batch, sh.n_heads, dh, S + 40)
        np.testing.assert_array_equal(raw[:, :, :, :S], kv8.to_bytes(fmt, ref.code[:, :, :, :S]))
        nb = -(-S // 32)
        np.testing.assert_array_equal(f64(kv[l].tensors[1]).reshape(ref.scale.shape)[..., :nb], ref.scale[..., :nb])


def _oracle_step(X, w64, caches, pos, n_heads, kind, active, eps=1e-5):
    """infer.decode with each active layer's keys and values, the new rows' among
    them, read from its 8-bit cache."""
    X = X.copy()
    B, n, d = X.shape
    for l, w in enumerate(w64):
        if not active[l]:
            continue
        w = {k: np.asarray(v, dtype=np.float64) for k, v in w.items()}
        qkv = np.stack([block.rmsnorm(X[b], w["g_attn"], eps)[0] @ w["w_qkv"].T for b in range(B)])
        qkv = qkv.reshape(B, n, 3, n_heads, d // n_heads)
        caches[l].store(qkv[:, :, 1:], pos)
        a, _, _ = kv8.attention(np.nan_to_num(caches[l].read()), qkv[:, :, 0], pos, kind == 1)
        for b in range(B):
            z = X[b] + a[b].reshape(n, d) @ w["w_o"].T
            X[b], _ = block.ffn_forward(z, w, 1.0, eps, kind)
    return X


@pytest.mark.parametrize("sh", SHAPES, ids=IDS)
@pytest.mark.parametrize("batch", [2, 5, 9])
@FMTS
def test_decode(sh, batch, fmt):
    """Full steps and drafts of one and several rows after a prefill, over up to
    72 rows (each of the projections' forms)."""
    sh = dataclasses.replace(sh, batch=batch, seq=64)
    dh = sh.d_model // sh.n_heads
    L, W = sh.n_layers, _weights(sh)
    wd, w64 = [w[0] for w in W], [w[1] for w in W]
    X = inp.hidden(dataclasses.replace(sh, seq=128))
    bf = [torch.zeros(batch, 64, 2 * sh.d_model, dtype=torch.bfloat16, device=DEV) for _ in range(L)]
    ld.ld_stack_eval(_cfg(sh), wd, X[:, :64].contiguous().to(DEV), _buf(ld.ld_eval_ws_bytes(_cfg(sh))), kv=bf, s_max=64)
    kv = _caches(sh, fmt, 16, 100)
    _prefill(sh, W, kv, X[:, :64].contiguous())
    refs = []
    for l in range(L):
        refs.append(kv8.Cache(fmt, 16, batch, sh.n_heads, dh, 100))
        refs[l].store(_split(bf[l], sh.n_heads), [0] * batch)
    full, draft = [1] * L, [1 if l % 2 == 0 else 0 for l in range(L)]
    ws = _buf(ld.ld_decode_kv8_ws_bytes(_cfg(sh), 8, 100))
    pos = 64
    for n, act in [(3, full), (1, draft), (2, full), (8, full), (1, full)]:
        x = X[:, pos:pos + n].contiguous()
        xd = x.to(DEV)
        ld.ld_stack_decode_kv8(_cfg(sh), wd, xd, [k if a else None for k, a in zip(kv, act)], pos, n, ws, active=act)
        want = _oracle_step(inp.f64(x), w64, refs, [pos] * batch, sh.n_heads, sh.kind, act)
        assert rel(f64(xd), want) < tol("bf16"), (pos, n, act)
        if act is full:
            pos += n


def test_decode_ragged_is_each_sequences():
    """seq_pos: a sequence's rows and caches bit for bit those of a step of all
    sequences at its position; sequences left out write nothing."""
    sh = dataclasses.replace(SMALL_BF16_128, batch=4, seq=128)
    L, W, n = sh.n_layers, _weights(sh), 3
    wd = [w[0] for w in W]
    cfg = _cfg(sh)
    kv = _caches(sh, kv8.E4M3, 64, 140)
    _prefill(sh, W, kv, inp.hidden(sh))
    x = inp.hidden(dataclasses.replace(sh, seq=n))
    ws = _buf(ld.ld_decode_kv8_ws_bytes(cfg, n, 140))
    pos = [128, 17, None, 64]
    mixed = _copy(kv)
    xm = x.to(DEV)
    sp = torch.tensor([-1 if p is None else p for p in pos], dtype=torch.int32, device=DEV)
    ld.ld_stack_decode_kv8(cfg, wd, xm, mixed, 128, n, ws, seq_pos=sp)
    for b, p in enumerate(pos):
        one = _copy(kv)
        xo = x.to(DEV)
        if p is not None:
            ld.ld_stack_decode_kv8(cfg, wd, xo, one, p, n, ws)
            assert torch.equal(xm[b], xo[b])
        for m, o in zip(mixed, one):
            for a, c in zip(m.tensors, o.tensors):
                a, c = (t.view(sh.batch, -1)[b] for t in (a, c))
                assert torch.equal(a.nan_to_num(7.0), c.nan_to_num(7.0)) if a.is_floating_point() else torch.equal(a, c)
    assert bool(torch.isfinite(xm).all())


def test_decode_captured():
    """One captured step decodes on as seq_pos advances, as eager steps do, with
    eager work of other sizes between the replays."""
    sh = dataclasses.replace(SMALL_BF16, batch=3, seq=64)
    L, W = sh.n_layers, _weights(sh)
    wd = [w[0] for w in W]
    cfg = _cfg(sh)
    base = _caches(sh, kv8.INT8, 32, 90)
    _prefill(sh, W, base, inp.hidden(sh))
    rows = inp.hidden(dataclasses.replace(sh, seq=128))[:, 64:]
    start = torch.tensor([64, 20, 33], dtype=torch.int32, device=DEV)

    def fresh():
        return [_copy(base), torch.zeros(sh.batch, 1, sh.d_model, dtype=torch.bfloat16, device=DEV), start.clone(),
                _buf(ld.ld_decode_kv8_ws_bytes(cfg, 1, 90))]

    def step(kv, x, sp, ws):
        ld.ld_stack_decode_kv8(cfg, wd, x, kv, 80, 1, ws, seq_pos=sp)
        sp += 1

    eager, cap = fresh(), fresh()
    step(*fresh())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(*cap)
    for i in range(6):
        for s in (eager, cap):
            s[1].copy_(rows[:, i:i + 1])
        step(*eager)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager[1], cap[1]) and torch.equal(eager[2], cap[2])
        for a, b in zip(eager[0], cap[0]):
            assert torch.equal(a.tensors[0], b.tensors[0])
        ld.ld_kv8_load(eager[0][0], 0, 7 + i, torch.zeros(3, 7 + i, 2 * sh.d_model, dtype=torch.bfloat16, device=DEV))
