"""Prefill and decoding of a stack over 4-bit caches, with bf16 and 4-bit weights
(ld_stack_eval_kv4, ld_stack_decode_kv4, ld_stack_decode_w4), against the float64
oracle."""
import dataclasses

import numpy as np
import pytest
import torch

import ld_inputs as inp
import paper_2609_05275_amd as ld
from oracle import block, kv4, kv8, w4
from tests.gpu_util import DEV, f64, layer_weights_dev, rel, tol
from tests.test_gpu_layer import SMALL_BF16, SMALL_BF16_128, SMALL_P, SMALL_P_128, _buf, _cfg

pytestmark = pytest.mark.gpu

SHAPES = [SMALL_BF16, SMALL_P, SMALL_BF16_128, SMALL_P_128]
IDS = ["small", "paper_small", "small_dh128", "paper_small_dh128"]
MATRICES = ("w_qkv", "w_o", "w_gate_up", "w_down")


def _caches(sh, s_max, sums=False):
    dh = sh.d_model // sh.n_heads
    out = []
    for _ in range(sh.n_layers):
        probe = ld.kv4(None, None, sh.batch, sh.n_heads, dh, s_max)
        codes = torch.full((ld.ld_kv4_code_bytes(probe),), 0xFF, dtype=torch.uint8, device=DEV)
        scales = torch.full((ld.ld_kv4_scale_bytes(probe),), 0xFF, dtype=torch.uint8, device=DEV)
        s = torch.full((sh.batch, sh.n_heads, s_max), 1e9, device=DEV) if sums else None
        out.append(ld.kv4(codes, scales, sh.batch, sh.n_heads, dh, s_max, sums=s))
    return out


def _copy(kv):
    return [ld.kv4(*[t.clone() for t in k.tensors[:2]], k.n_seq, k.n_kv_heads, k.d_head, k.s_max,
                   sums=None if k.tensors[2] is None else k.tensors[2].clone()) for k in kv]


def _weights(sh):
    return [layer_weights_dev(sh, l, gain_jitter=True) for l in range(sh.n_layers)]


def _in_4_bits(sh, W, formats):
    """Device weights in 4 bits, matrix i of a layer in formats[i], and their values."""
    out = []
    for wd, w64 in W:
        d, v = dict(wd), dict(w64)
        for name, (fmt, group) in zip(MATRICES, formats):
            n, k = w64[name].shape
            probe = ld.w4(None, None, fmt, group, n, k)
            scales = torch.zeros(ld.ld_w4_scale_bytes(probe), dtype=torch.uint8, device=DEV)
            d[name] = ld.w4(torch.zeros(ld.ld_w4_code_bytes(probe), dtype=torch.uint8, device=DEV),
                            scales if fmt == w4.E2M1 else scales.view(torch.bfloat16), fmt, group, n, k)
            ld.ld_w4_pack(d[name], wd[name])
            v[name] = w4.values(fmt, group, w64[name])
        out.append((d, v))
    return out


def _prefill(sh, W, kv, x, active=None):
    xd = x.to(DEV)
    ld.ld_stack_eval_kv4(_cfg(sh), [w[0] for w in W], xd, _buf(ld.ld_eval_ws_bytes(_cfg(sh))), kv, active=active)
    return xd


def _split(kv, n_heads):
    """A bf16 cache [B, S, 2 d] as rows [B, S, 2, H, dh] in float64."""
    B, S, d2 = kv.shape
    return f64(kv).reshape(B, S, 2, n_heads, d2 // 2 // n_heads)


@pytest.mark.parametrize("sh", SHAPES, ids=IDS)
def test_prefill(sh):
    """Hidden states bit for bit ld_stack_eval's; caches the oracle's codes of the keys
    and values it stores; skipped layers' caches untouched."""
    L, S = sh.n_layers, sh.seq
    act = [1] * (L - 1) + [0]
    W, x = _weights(sh), inp.hidden(sh)
    cfg = _cfg(sh)
    want = x.to(DEV)
    bf = [torch.zeros(sh.batch, S, 2 * sh.d_model, dtype=torch.bfloat16, device=DEV) for _ in range(L)]
    ld.ld_stack_eval(cfg, [w[0] for w in W], want, _buf(ld.ld_eval_ws_bytes(cfg)), active=act, kv=bf, s_max=S)
    kv = _caches(sh, S + 40, sums=True)
    kv[-1] = None
    got = _prefill(sh, W, kv, x, active=act)
    assert torch.equal(got, want)
    dh = sh.d_model // sh.n_heads
    for l in range(L - 1):
        ref = kv4.Cache(sh.batch, sh.n_heads, dh, S + 40)
        ref.store(_split(bf[l], sh.n_heads), [0] * sh.batch)
        raw = kv4.unpack(kv[l].tensors[0].cpu().numpy(), sh.batch, sh.n_heads, dh, S + 40)[..., :S, :]
        np.testing.assert_array_equal(kv4.from_codes(raw), ref.code[..., :S, :])
        sc = kv[l].tensors[1].cpu().numpy().reshape(sh.batch, sh.n_heads, 2, -1, dh // 32)
        np.testing.assert_array_equal(sc[..., :S, :], ref.scale[..., :S, :])
        assert not bool(kv[l].tensors[2][..., :S].any()) and bool((kv[l].tensors[2][..., S:] == 1e9).all())


def _oracle_step(X, w64, caches, pos, n_heads, kind, active, eps=1e-5):
    """infer.decode with each active layer's keys and values, the new rows' among
    them, read from its 4-bit cache, whose sums take the weights."""
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
        caches[l].sums += kv4.weights(caches[l].read(), qkv[:, :, 0], pos, kind == 1)
        for b in range(B):
            z = X[b] + a[b].reshape(n, d) @ w["w_o"].T
            X[b], _ = block.ffn_forward(z, w, 1.0, eps, kind)
    return X


def _adopt(kv, ref, pos, n):
    """The new rows' codes as the GPU rounded them (a code may fall to either side where
    the projection's own rounding decides), after a check that they are near."""
    dh = kv.d_head
    code = kv4.from_codes(kv4.unpack(kv.tensors[0].cpu().numpy(), kv.n_seq, kv.n_kv_heads, dh, kv.s_max))[..., pos:pos + n, :]
    sc = kv.tensors[1].cpu().numpy().reshape(kv.n_seq, kv.n_kv_heads, 2, -1, dh // 32)[..., pos:pos + n, :]
    got = code * np.repeat(kv4.scale_of(sc), 32, -1)
    want = ref.read()[..., pos:pos + n, :]
    # where a code or a scale falls to the other side it is off by a step, 2 of 6 at most twice over
    top = np.abs(want).reshape(*want.shape[:-1], -1, 32).max(-1).repeat(32, -1)
    assert np.all(np.abs(got - want) <= 0.7 * top) and np.mean(got != want) < 0.1
    ref.code[..., pos:pos + n, :], ref.scale[..., pos:pos + n, :] = code, sc


@pytest.mark.parametrize("sh", SHAPES, ids=IDS)
@pytest.mark.parametrize("batch", [2, 5, 9])
@pytest.mark.parametrize("four", [False, True], ids=["bf16", "w4"])
def test_decode(sh, batch, four):
    """Full steps and drafts of one and several rows after a prefill, over up to 72
    rows, in bf16 and 4-bit weights of mixed formats; the sums of the caches."""
    sh = dataclasses.replace(sh, batch=batch, seq=64)
    dh = sh.d_model // sh.n_heads
    L, W = sh.n_layers, _weights(sh)
    if four:
        V = _in_4_bits(sh, W, [(w4.E2M1, 32), (w4.INT4, 32), (w4.INT4, 64), (w4.INT4, 128)])
        # a prefill in bf16 by what the 4 bits stand for (rounded to bf16)
        W = [({k: torch.from_numpy(np.asarray(v)).to(torch.bfloat16).to(DEV) for k, v in v64.items()}, v64) for _, v64 in V]
        wd, w64 = [v[0] for v in V], [v[1] for v in V]
        step = ld.ld_stack_decode_w4
    else:
        wd, w64 = [w[0] for w in W], [w[1] for w in W]
        step = ld.ld_stack_decode_kv4
    X = inp.hidden(dataclasses.replace(sh, seq=128))
    bf = [torch.zeros(batch, 64, 2 * sh.d_model, dtype=torch.bfloat16, device=DEV) for _ in range(L)]
    ld.ld_stack_eval(_cfg(sh), [w[0] for w in W], X[:, :64].contiguous().to(DEV), _buf(ld.ld_eval_ws_bytes(_cfg(sh))), kv=bf, s_max=64)
    kv = _caches(sh, 100, sums=True)
    _prefill(sh, W, kv, X[:, :64].contiguous())
    refs = []
    for l in range(L):
        refs.append(kv4.Cache(batch, sh.n_heads, dh, 100))
        refs[l].store(_split(bf[l], sh.n_heads), [0] * batch)
    full, draft = [1] * L, [1 if l % 2 == 0 else 0 for l in range(L)]
    ws = _buf(ld.ld_decode_kv4_ws_bytes(_cfg(sh), 8, 100, sums=True))
    pos = 64
    for n, act in [(3, full), (1, draft), (2, full), (8, full), (1, full)]:
        x = X[:, pos:pos + n].contiguous()
        xd = x.to(DEV)
        step(_cfg(sh), wd, xd, [k if a else None for k, a in zip(kv, act)], pos, n, ws, active=act)
        want = _oracle_step(inp.f64(x), w64, refs, [pos] * batch, sh.n_heads, sh.kind, act)
        # a code that falls to the other side moves a row's attention by a step of one of its values
        assert rel(f64(xd), want) < 1.5 * tol("bf16"), (pos, n, act)
        for l in range(L):
            if act[l]:
                _adopt(kv[l], refs[l], pos, n)
                # a weight's relative error is its score's error: the queries' and keys' bf16, some 2^-7 of scores of a few
                assert rel(f64(kv[l].tensors[2][..., :pos + n]), refs[l].sums[..., :pos + n]) < 0.05
        if act is full:
            pos += n


def test_decode_ragged_is_each_sequences():
    """seq_pos: a sequence's rows, caches and sums bit for bit those of a step of all
    sequences at its position; sequences left out write nothing."""
    sh = dataclasses.replace(SMALL_BF16_128, batch=4, seq=128)
    L, W, n = sh.n_layers, _weights(sh), 3
    V = _in_4_bits(sh, W, [(w4.INT4, 64)] * 4)
    cfg = _cfg(sh)
    kv = _caches(sh, 140, sums=True)
    _prefill(sh, W, kv, inp.hidden(sh))
    x = inp.hidden(dataclasses.replace(sh, seq=n))
    ws = _buf(ld.ld_decode_kv4_ws_bytes(cfg, n, 140, sums=True))
    pos = [128, 17, None, 64]
    sp = torch.tensor([-1 if p is None else p for p in pos], dtype=torch.int32, device=DEV)
    for step, wd in ((ld.ld_stack_decode_kv4, [w[0] for w in W]), (ld.ld_stack_decode_w4, [v[0] for v in V])):
        mixed, xm = _copy(kv), x.to(DEV)
        step(cfg, wd, xm, mixed, 128, n, ws, seq_pos=sp)
        for b, p in enumerate(pos):
            one, xo = _copy(kv), x.to(DEV)
            if p is not None:
                step(cfg, wd, xo, one, p, n, ws)
                assert torch.equal(xm[b], xo[b])
            for m, o in zip(mixed, one):
                for a, c in zip(m.tensors, o.tensors):
                    assert torch.equal(a.view(sh.batch, -1)[b], c.view(sh.batch, -1)[b])
        assert bool(torch.isfinite(xm).all())


def test_drafts_leave_no_mark():
    """A draft's rows, then the verify step over them: the caches bit for bit those of a
    verify step without a draft."""
    sh = dataclasses.replace(SMALL_BF16, batch=2, seq=64)
    W = _weights(sh)
    V = _in_4_bits(sh, W, [(w4.E2M1, 32)] * 4)
    wd, cfg = [v[0] for v in V], _cfg(sh)
    kv = _caches(sh, 90)
    _prefill(sh, W, kv, inp.hidden(sh))
    x = inp.hidden(dataclasses.replace(sh, seq=128))[:, 64:69].contiguous()
    ws = _buf(ld.ld_decode_kv4_ws_bytes(cfg, 8, 90))
    plain, drafted = _copy(kv), _copy(kv)
    for i in range(4):
        ld.ld_stack_decode_w4(cfg, wd, (100 * x[:, i:i + 1]).contiguous().to(DEV), drafted, 64 + i, 1, ws,
                              active=[1] + [0] * (sh.n_layers - 1))
    got, want = x.to(DEV), x.to(DEV)
    ld.ld_stack_decode_w4(cfg, wd, got, drafted, 64, 5, ws)
    ld.ld_stack_decode_w4(cfg, wd, want, plain, 64, 5, ws)
    assert torch.equal(got, want)
    for a, b in zip(drafted, plain):
        assert torch.equal(a.tensors[0], b.tensors[0]) and torch.equal(a.tensors[1], b.tensors[1])


def test_decode_captured():
    """One captured step decodes on as seq_pos advances, as eager steps do, with
    eager work of other sizes between the replays."""
    sh = dataclasses.replace(SMALL_BF16, batch=3, seq=64)
    L, W = sh.n_layers, _weights(sh)
    V = _in_4_bits(sh, W, [(w4.INT4, 32)] * 4)
    wd, cfg = [v[0] for v in V], _cfg(sh)
    base = _caches(sh, 90, sums=True)
    _prefill(sh, W, base, inp.hidden(sh))
    for k in base:
        k.tensors[2].zero_()
    rows = inp.hidden(dataclasses.replace(sh, seq=128))[:, 64:]
    start = torch.tensor([64, 20, 33], dtype=torch.int32, device=DEV)

    def fresh():
        return [_copy(base), torch.zeros(sh.batch, 1, sh.d_model, dtype=torch.bfloat16, device=DEV), start.clone(),
                _buf(ld.ld_decode_kv4_ws_bytes(cfg, 1, 90, sums=True))]

    def step(kv, x, sp, ws):
        ld.ld_stack_decode_w4(cfg, wd, x, kv, 80, 1, ws, seq_pos=sp)
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
            assert all(torch.equal(s, t) for s, t in zip(a.tensors, b.tensors))
        ld.ld_kv4_load(eager[0][0], 0, 7 + i, torch.zeros(3, 7 + i, 2 * sh.d_model, dtype=torch.bfloat16, device=DEV))
