"""What the stack calls over 8-bit caches refuse (no GPU: nothing here reaches
the HIP runtime)."""
import pytest
import torch

import paper_2609_05275_amd as ld
from tests.test_abi_kv8 import INVALID, SHAPE, UNSUPPORTED, WORKSPACE, Raw

P = 1 << 20
W = [{k: P for k in ld.WEIGHT_KEYS}] * 2
WS = Raw(P)


def cfg(**kw):
    return ld.config(**{**dict(batch=2, seq=64, d_model=256, n_heads=2, d_ff=512, dtype=ld.LD_BF16), **kw})


def desc(**kw):
    k = ld.ld_kv8(**{**dict(format=0, block=64, n_seq=2, n_kv_heads=2, d_head=128, s_max=100), **kw})
    k.codes, k.scales = kw.get("codes", P), kw.get("scales", P)
    return k


def evaluate(c=None, kv=None, ws=WS, x=P):
    ld.ld_stack_eval_kv8(c or cfg(), W, x, ws, kv or [desc(), desc()], stream=0)


def decode(c=None, kv=None, ws=WS, x=P, pos=64, n=1, seq_pos=None, active=None):
    ld.ld_stack_decode_kv8(c or cfg(), W, x, kv or [desc(), desc()], pos, n, ws, seq_pos=seq_pos, active=active, stream=0)


@pytest.mark.parametrize("kw,code", [(dict(n_seq=3), SHAPE), (dict(n_kv_heads=1), SHAPE), (dict(d_head=64), SHAPE),
                                     (dict(format=7), INVALID), (dict(block=40), UNSUPPORTED), (dict(s_max=63), SHAPE)])
def test_descriptor_against_the_configuration(kw, code):
    for call in (evaluate, decode):
        with pytest.raises(ld.LdError) as e:
            call(kv=[desc(), desc(**kw)])
        assert e.value.status == code


def test_null_buffers():
    bad = desc()
    bad.scales = None
    for call in (evaluate, decode):
        with pytest.raises(ld.LdError) as e:
            call(kv=[desc(), bad])
        assert e.value.status == INVALID
        with pytest.raises(ld.LdError) as e:
            call(kv=[desc(), None])          # a missing cache of an active layer
        assert e.value.status != 0


@pytest.mark.parametrize("kw,code", [(dict(n=0), INVALID), (dict(n=9), INVALID), (dict(pos=-1), SHAPE),
                                     (dict(pos=100), SHAPE), (dict(pos=2 ** 31 - 1), SHAPE), (dict(x=None), INVALID),
                                     (dict(seq_pos=Raw(P + 2)), INVALID), (dict(ws=Raw(P, 1000)), WORKSPACE)])
def test_decode_arguments(kw, code):
    with pytest.raises(ld.LdError) as e:
        decode(**kw)
    assert e.value.status == code


def test_types_and_workspaces():
    f32 = cfg(dtype=ld.LD_F32, d_model=128, n_heads=2)
    for call in (evaluate, decode):
        with pytest.raises(ld.LdError) as e:
            call(c=f32, kv=[desc(d_head=64)] * 2)
        assert e.value.status == UNSUPPORTED
    with pytest.raises(ld.LdError) as e:
        evaluate(ws=Raw(P, 1000))
    assert e.value.status == WORKSPACE
    last = 0
    for s_max in (1, 100, 1000, 5000, 100000):
        n = ld.ld_decode_kv8_ws_bytes(cfg(), 3, s_max)
        assert n >= last > -1
        last = n
    assert ld.ld_decode_kv8_ws_bytes(cfg(), 0, 10) == ld.ld_decode_kv8_ws_bytes(cfg(), 9, 10) == 0
    assert ld.ld_decode_kv8_ws_bytes(cfg(), 1, 0) == ld.ld_decode_kv8_ws_bytes(cfg(n_heads=3), 1, 10) == 0


def test_null_array():
    lib = ld._lib
    import ctypes as C
    c = cfg()
    w = (ld.ld_weights * 2)(*[ld.weights(x) for x in W])
    p = C.c_void_p(P)
    assert lib.ld_stack_eval_kv8(C.byref(c), 2, w, None, None, p, None, p, 1 << 40, None) == INVALID
    assert lib.ld_stack_decode_kv8(C.byref(c), 2, w, None, None, p, None, 0, None, 1, p, 1 << 40, None) == INVALID


def test_binding():
    with pytest.raises(ValueError, match="layers"):
        evaluate(kv=[desc()])
    with pytest.raises(ValueError, match="x:"):
        decode(x=torch.zeros(2, 2, 256, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="seq_pos"):
        decode(seq_pos=torch.zeros(2, dtype=torch.int64))
