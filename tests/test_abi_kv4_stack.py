"""What the stack calls over 4-bit caches and weights refuse (no GPU: nothing here
reaches the HIP runtime)."""
import ctypes as C

import pytest
import torch

import paper_2609_05275_amd as ld
from tests.test_abi_kv8 import INVALID, SHAPE, UNSUPPORTED, WORKSPACE, Raw
from tests.test_abi_kv8_binding import elsewhere

P = 1 << 20
W = [{k: P for k in ld.WEIGHT_KEYS}] * 2
WS = Raw(P)


def cfg(**kw):
    return ld.config(**{**dict(batch=2, seq=64, d_model=256, n_heads=2, d_ff=512, dtype=ld.LD_BF16), **kw})


def desc(**kw):
    k = ld.ld_kv4(**{**dict(n_seq=2, n_kv_heads=2, d_head=128, s_max=100), **{a: b for a, b in kw.items() if a != "sums"}})
    k.codes, k.scales, k.sums = P, P, kw.get("sums")
    return k


def w4(n, k, **kw):
    w = ld.ld_w4(kw.get("format", 1), kw.get("group", 64), n, k)
    w.codes, w.scales = kw.get("codes", P), kw.get("scales", P)
    return w


def weights(**kw):
    w = dict(g_attn=P, g_mlp=P, w_qkv=w4(768, 256), w_o=w4(256, 256), w_gate_up=w4(1024, 256), w_down=w4(256, 512))
    return {**w, **kw}


def evaluate(c=None, kv=None, ws=WS, x=P):
    ld.ld_stack_eval_kv4(c or cfg(), W, x, ws, kv or [desc(), desc()], stream=0)


def decode(c=None, kv=None, ws=WS, x=P, pos=64, n=1, seq_pos=None, active=None):
    ld.ld_stack_decode_kv4(c or cfg(), W, x, kv or [desc(), desc()], pos, n, ws, seq_pos=seq_pos, active=active, stream=0)


def decode_w4(c=None, kv=None, ws=WS, x=P, pos=64, n=1, seq_pos=None, active=None, w=None):
    ld.ld_stack_decode_w4(c or cfg(), w or [weights()] * 2, x, kv or [desc(), desc()], pos, n, ws, seq_pos=seq_pos,
                          active=active, stream=0)


CALLS = (evaluate, decode, decode_w4)


@pytest.mark.parametrize("kw,code", [(dict(n_seq=3), SHAPE), (dict(n_kv_heads=1), SHAPE), (dict(d_head=64), SHAPE),
                                     (dict(d_head=96), UNSUPPORTED), (dict(s_max=63), SHAPE)], ids=str)
def test_descriptor_against_the_configuration(kw, code):
    for call in CALLS:
        with pytest.raises(ld.LdError) as e:
            call(kv=[desc(), desc(**kw)])
        assert e.value.status == code


def test_null_buffers():
    bad = desc()
    bad.scales = None
    for call in CALLS:
        with pytest.raises(ld.LdError) as e:
            call(kv=[desc(), bad])
        assert e.value.status == INVALID
        with pytest.raises(ld.LdError) as e:
            call(kv=[desc(), None])          # a missing cache of an active layer
        assert e.value.status != 0


@pytest.mark.parametrize("kw,code", [(dict(n=0), INVALID), (dict(n=9), INVALID), (dict(pos=-1), SHAPE),
                                     (dict(pos=100), SHAPE), (dict(pos=2 ** 31 - 1), SHAPE), (dict(x=None), INVALID),
                                     (dict(seq_pos=Raw(P + 2)), INVALID), (dict(ws=Raw(P, 1000)), WORKSPACE),
                                     (dict(ws=None), INVALID)],
                         ids=["no rows", "nine rows", "pos", "pos at the end", "pos beyond 32 bits", "no x", "seq_pos", "little ws", "no ws"])
def test_decode_arguments(kw, code):
    for call in (decode, decode_w4):
        with pytest.raises(ld.LdError) as e:
            call(**kw)
        assert e.value.status == code


BAD_W = [(dict(g_attn=None), INVALID), (dict(g_mlp=P + 2), INVALID), (dict(w_qkv=w4(256, 256)), SHAPE),
         (dict(w_o=w4(256, 512)), SHAPE), (dict(w_gate_up=w4(512, 256)), SHAPE), (dict(w_down=w4(256, 256)), SHAPE),
         (dict(w_o=w4(256, 256, codes=None)), INVALID), (dict(w_o=w4(256, 256, scales=P + 8)), INVALID),
         (dict(w_o=w4(256, 256, format=4)), INVALID), (dict(w_o=w4(256, 256, group=8)), UNSUPPORTED)]


@pytest.mark.parametrize("kw,code", BAD_W, ids=[f"{next(iter(k))}-{i}" for i, (k, _) in enumerate(BAD_W)])
def test_weights(kw, code):
    with pytest.raises(ld.LdError) as e:
        decode_w4(w=[weights(), weights(**kw)])
    assert e.value.status == code


def test_squared_relu_weights():
    """One matrix of d_ff rows instead of two."""
    with pytest.raises(ld.LdError) as e:
        decode_w4(c=cfg(block_kind=1))
    assert e.value.status == SHAPE


def test_sums_need_more_scratch():
    n = ld.ld_decode_kv4_ws_bytes(cfg(), 1, 100)
    assert ld.ld_decode_kv4_ws_bytes(cfg(), 1, 100, sums=True) >= n + 2 * 2 * 100 * 4
    for call in (decode, decode_w4):
        with pytest.raises(ld.LdError) as e:
            call(kv=[desc(), desc(sums=P)], ws=Raw(P, n))
        assert e.value.status == WORKSPACE


def test_types_and_workspaces():
    f32 = cfg(dtype=ld.LD_F32, d_model=128, n_heads=2)
    for call in CALLS:
        with pytest.raises(ld.LdError) as e:
            call(c=f32, kv=[desc(d_head=64)] * 2)
        assert e.value.status == UNSUPPORTED
    for sums in (False, True):
        last = 0
        for s_max in (1, 100, 1000, 5000, 100000):
            n = ld.ld_decode_kv4_ws_bytes(cfg(), 3, s_max, sums)
            assert n >= last > -1
            last = n
        n = [ld.ld_decode_kv4_ws_bytes(cfg(batch=9, d_model=512, n_heads=4), i, 300, sums) for i in range(1, 9)]
        assert n == sorted(n)
    assert ld.ld_decode_kv4_ws_bytes(cfg(), 0, 10) == ld.ld_decode_kv4_ws_bytes(cfg(), 9, 10) == 0
    assert ld.ld_decode_kv4_ws_bytes(cfg(), 1, 0) == ld.ld_decode_kv4_ws_bytes(cfg(n_heads=3), 1, 10) == 0


def test_null_arrays():
    lib, c, p = ld._lib, cfg(), C.c_void_p(P)
    w = (ld.ld_weights * 2)(*[ld.weights(x) for x in W])
    k = (ld.ld_kv4 * 2)(desc(), desc())
    assert lib.ld_stack_eval_kv4(C.byref(c), 2, w, None, None, p, None, p, 1 << 40, None) == INVALID
    assert lib.ld_stack_decode_kv4(C.byref(c), 2, w, None, None, p, None, 0, None, 1, p, 1 << 40, None) == INVALID
    assert lib.ld_stack_decode_kv4(C.byref(c), 2, None, None, None, p, k, 0, None, 1, p, 1 << 40, None) == INVALID
    assert lib.ld_stack_decode_w4(C.byref(c), 2, None, None, None, p, k, 0, None, 1, p, 1 << 40, None) == INVALID


def test_binding(monkeypatch):
    for call in CALLS:
        with pytest.raises(ValueError, match="layers"):
            call(kv=[desc()])
        with pytest.raises(ValueError, match="x:"):
            call(x=torch.zeros(2, 2, 256, dtype=torch.bfloat16))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for call in (decode, decode_w4):
        with pytest.raises(ValueError, match="seq_pos"):
            call(seq_pos=torch.zeros(2, dtype=torch.int64))
        with pytest.raises(ValueError, match="current device"):
            call(x=elsewhere(2, 1, 256))
    far = weights()
    far["w_down"].device = 1
    with pytest.raises(ValueError, match="current device"):
        decode_w4(w=[far, weights()])
