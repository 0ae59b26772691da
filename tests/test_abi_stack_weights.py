"""What the stack calls refuse in the weights they are given: another type than the
configuration's, or another number of elements (no GPU: nothing here reaches the HIP
runtime)."""
import pytest
import torch

import paper_2609_05275_amd as ld
from tests.test_abi_kv4_stack import P, WS, cfg, decode_w4, desc, weights
from tests.test_abi_kv8 import Raw
from tests.test_abi_kv8_binding import elsewhere
from tests.test_abi_kv8_stack import desc as desc8

SIZES = dict(g_attn=256, w_qkv=768 * 256, w_o=256 * 256, g_mlp=256, w_gate_up=1024 * 256, w_down=256 * 512)
PLAIN = {k: P for k in ld.WEIGHT_KEYS}


def evaluate(w, **kw):
    ld.ld_stack_eval(cfg(), w, P, WS, stream=0, **kw)


def decode(w, **kw):
    ld.ld_stack_decode(cfg(), w, P, [Raw(P)] * 2, 100, 64, 1, WS, stream=0, **kw)


def evaluate_kv8(w, **kw):
    ld.ld_stack_eval_kv8(cfg(), w, P, WS, [desc8()] * 2, stream=0, **kw)


def decode_kv8(w, **kw):
    ld.ld_stack_decode_kv8(cfg(), w, P, [desc8()] * 2, 64, 1, WS, stream=0, **kw)


def evaluate_kv4(w, **kw):
    ld.ld_stack_eval_kv4(cfg(), w, P, WS, [desc()] * 2, stream=0, **kw)


def decode_kv4(w, **kw):
    ld.ld_stack_decode_kv4(cfg(), w, P, [desc()] * 2, 64, 1, WS, stream=0, **kw)


OLDER = (evaluate, decode)
OVER_CACHES = (evaluate_kv8, decode_kv8, evaluate_kv4, decode_kv4)


@pytest.mark.parametrize("call", OLDER + OVER_CACHES, ids=lambda c: c.__name__)
@pytest.mark.parametrize("key", ld.WEIGHT_KEYS)
def test_type_and_size(call, key):
    for t in (elsewhere(SIZES[key], dtype=torch.float32), elsewhere(SIZES[key] - 1), elsewhere(SIZES[key] + 8)):
        with pytest.raises(ValueError, match=f"^{key}: (dtype|[0-9]+ elements)"):
            call([PLAIN, {**PLAIN, key: t}])


@pytest.mark.parametrize("call", OVER_CACHES, ids=lambda c: c.__name__)
def test_device(call, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="w_o: .*current device"):
        call([PLAIN, {**PLAIN, "w_o": elsewhere(256 * 256)}])


@pytest.mark.parametrize("key", ["g_attn", "g_mlp"])
def test_gains_of_4_bit_weights(key, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for t, what in ((elsewhere(256, dtype=torch.float32), "dtype"), (elsewhere(255), "255 elements"),
                    (elsewhere(512), "512 elements"), (elsewhere(256), ".*current device"),
                    (torch.zeros(256, dtype=torch.bfloat16), "a device tensor")):
        with pytest.raises(ValueError, match=f"^{key}: {what}"):
            decode_w4(w=[weights(), weights(**{key: t})])


def test_a_skipped_layer_is_not_looked_at():
    """The active set may come from a generator."""
    w = [PLAIN, {**PLAIN, "g_attn": elsewhere(8)}]
    for call in OLDER + OVER_CACHES:
        with pytest.raises(ld.LdError, match=r"r_eval\[0\]"):
            call(w, active=(a for a in (1, 0)), r_eval=[float("nan")] * 2)
