"""What the 4-bit cache's calls refuse, and its sizes (no GPU: no call here
reaches the HIP runtime)."""
import ctypes as C

import pytest
import torch

import paper_2609_05275_amd as ld
from tests.test_abi_kv8 import INVALID, SHAPE, UNSUPPORTED, WORKSPACE, OnDevice, Raw

P = 1 << 20
A = Raw(P)
GOOD = dict(n_seq=2, n_kv_heads=4, d_head=128, s_max=100)


def desc(codes=P, scales=P, sums=None, **kw):
    kv = ld.ld_kv4(**{**GOOD, **kw})
    kv.codes, kv.scales, kv.sums = codes, scales, sums
    return kv


def store(kv, n_heads=8, n_new=3, pos=5, qkv=A, seq_pos=None):
    ld.ld_kv4_store(kv, n_heads, n_new, pos, qkv, seq_pos=seq_pos, stream=0)


def load(kv, pos=5, n=3, out=A, seq_len=None):
    ld.ld_kv4_load(kv, pos, n, out, seq_len=seq_len, stream=0)


def attn(kv, n_heads=8, pos=5, n_new=3, qkv=A, o=A, ws=A, seq_pos=None, alibi=0):
    ld.ld_attn_decode_kv4(kv, n_heads, pos, n_new, qkv, o, ws, seq_pos=seq_pos, alibi=alibi, stream=0)


def evict(kv, to=None, length=90, keep=40, recent=5, idx=A, ws=A, seq_len=None):
    if to is None:
        to = desc(1 << 30, 1 << 31, 1 << 32, s_max=50)
    ld.ld_kv4_evict(kv, to, length, keep, recent, idx, ws, seq_len=seq_len, stream=0)


CALLS = (store, load, attn, evict)
BAD_DESC = [(dict(d_head=96), UNSUPPORTED), (dict(d_head=256), UNSUPPORTED), (dict(n_seq=0), SHAPE),
            (dict(n_kv_heads=0), SHAPE), (dict(s_max=0), SHAPE), (dict(n_seq=65536), SHAPE),
            (dict(n_kv_heads=32768), SHAPE), (dict(s_max=2 ** 31 - 1), SHAPE),
            (dict(n_seq=1, n_kv_heads=1, s_max=2 ** 30 + 1), SHAPE), (dict(n_seq=60000, n_kv_heads=30000), SHAPE)]


@pytest.mark.parametrize("kw,code", BAD_DESC, ids=[str(k) for k, _ in BAD_DESC])
def test_descriptor_refused(kw, code):
    kv = desc(sums=P, **kw)
    assert ld.ld_kv4_code_bytes(kv) == 0 and ld.ld_kv4_scale_bytes(kv) == 0
    assert ld.ld_attn_decode_kv4_ws_bytes(kv, 8, 1) == 0 and ld.ld_kv4_evict_ws_bytes(kv, 1, 1) == 0
    for call in CALLS:
        with pytest.raises(ld.LdError) as e:
            call(kv)
        assert e.value.status == code
    with pytest.raises(ld.LdError) as e:
        evict(desc(sums=P), to=kv)
    assert e.value.status == code


BAD_BUFFERS = [dict(codes=None), dict(scales=None), dict(codes=P + 8), dict(scales=P + 8), dict(sums=P + 2)]


@pytest.mark.parametrize("kw", BAD_BUFFERS, ids=[str(k) for k in BAD_BUFFERS])
def test_buffers_refused(kw):
    for call in CALLS:
        with pytest.raises(ld.LdError) as e:
            call(desc(**{"sums": P, **kw}))
        assert e.value.status == INVALID


OFF, NULL = Raw(P + 8), None
BAD_CALLS = [
    (store, dict(n_heads=6), SHAPE), (store, dict(n_heads=0), SHAPE), (store, dict(n_heads=65536), SHAPE),
    (store, dict(n_new=0), SHAPE), (store, dict(pos=-1), SHAPE), (store, dict(pos=98), SHAPE),
    (store, dict(pos=2 ** 31 - 1), SHAPE), (store, dict(qkv=NULL), INVALID), (store, dict(qkv=OFF), INVALID),
    (store, dict(seq_pos=Raw(P + 2)), INVALID),
    (load, dict(n=0), SHAPE), (load, dict(pos=-1), SHAPE), (load, dict(pos=98), SHAPE), (load, dict(out=NULL), INVALID),
    (load, dict(out=OFF), INVALID), (load, dict(seq_len=Raw(P + 2)), INVALID),
    (attn, dict(n_heads=6), SHAPE), (attn, dict(n_new=0), INVALID), (attn, dict(n_new=9), INVALID),
    (attn, dict(alibi=2), INVALID), (attn, dict(pos=-1), SHAPE), (attn, dict(pos=98), SHAPE),
    (attn, dict(qkv=NULL), INVALID), (attn, dict(o=NULL), INVALID), (attn, dict(qkv=OFF), INVALID),
    (attn, dict(o=Raw(P + 1)), INVALID), (attn, dict(ws=Raw(P + 4)), INVALID), (attn, dict(ws=Raw(P, 64)), WORKSPACE),
    (attn, dict(ws=None), INVALID), (attn, dict(seq_pos=Raw(P + 1)), INVALID),
    (evict, dict(length=0), SHAPE), (evict, dict(length=101), SHAPE), (evict, dict(keep=0), SHAPE),
    (evict, dict(keep=51), SHAPE), (evict, dict(recent=-1), SHAPE), (evict, dict(recent=41), SHAPE),
    (evict, dict(idx=NULL), INVALID), (evict, dict(idx=Raw(P + 2)), INVALID), (evict, dict(seq_len=Raw(P + 2)), INVALID),
    (evict, dict(to=desc(1 << 30, 1 << 31, n_seq=3)), SHAPE), (evict, dict(to=desc(1 << 30, 1 << 31, n_kv_heads=2)), SHAPE),
    (evict, dict(to=desc(1 << 30, 1 << 31, d_head=64)), SHAPE), (evict, dict(to=desc()), INVALID),
    (evict, dict(to=desc(1 << 30, 1 << 31, P + 4)), INVALID),
]


@pytest.mark.parametrize("call,kw,code", BAD_CALLS, ids=[f"{c.__name__}-{next(iter(k))}-{i}" for i, (c, k, _) in enumerate(BAD_CALLS)])
def test_call_refused(call, kw, code):
    with pytest.raises(ld.LdError) as e:
        call(desc(sums=P), **kw)
    assert e.value.status == code and ld.last_error()


def test_evict_needs_sums():
    with pytest.raises(ld.LdError) as e:
        evict(desc())
    assert e.value.status == INVALID


@pytest.mark.parametrize("which", ["codes", "scales", "sums"])
@pytest.mark.parametrize("end", [0, 1])
def test_evict_refuses_shared_memory(which, end):
    """The first or the last bytes of a buffer of one cache in one of the other."""
    fro = desc(1 << 30, 1 << 31, 1 << 32)
    n = {"codes": ld.ld_kv4_code_bytes(fro), "scales": ld.ld_kv4_scale_bytes(fro), "sums": 2 * 4 * 100 * 4}
    to = desc(1 << 33, 1 << 34, 1 << 35, s_max=50)
    at = getattr(fro, which) + (n[which] - 16 if end else 0)
    to.codes = at
    with pytest.raises(ld.LdError) as e:
        evict(fro, to=to)
    assert e.value.status == INVALID and "share" in ld.last_error()


def test_null_descriptor():
    lib, p = ld._lib, C.c_void_p(P)
    assert lib.ld_kv4_code_bytes(None) == lib.ld_kv4_scale_bytes(None) == 0
    assert lib.ld_kv4_store(None, 8, 1, 0, None, p, None) == INVALID
    assert lib.ld_kv4_load(None, 0, 1, None, p, None) == INVALID
    assert lib.ld_attn_decode_kv4(None, 8, 0, 0, None, 1, p, p, p, 1 << 30, None) == INVALID
    kv = desc(sums=P)
    assert lib.ld_kv4_evict(None, C.byref(kv), 1, None, 1, 0, p, p, 1 << 30, None) == INVALID
    assert lib.ld_kv4_evict(C.byref(kv), None, 1, None, 1, 0, p, p, 1 << 30, None) == INVALID


def test_sizes():
    kv = desc()
    assert ld.ld_kv4_code_bytes(kv) == 2 * 4 * 104 * 128            # 100 positions in 104
    assert ld.ld_kv4_scale_bytes(kv) == 2 * 4 * 2 * 104 * 4
    big = desc(n_seq=64, n_kv_heads=32, s_max=131072)               # past 32 bits
    assert ld.ld_kv4_code_bytes(big) == 64 * 32 * 131072 * 128
    for sums in (None, P):
        last = 0
        for s_max in (1, 64, 65, 256, 300, 1000, 4096, 70000, 131072):
            n = ld.ld_attn_decode_kv4_ws_bytes(desc(n_seq=1, s_max=s_max, sums=sums), 8, 3)
            assert n >= last > -1
            last = n
        n = [ld.ld_attn_decode_kv4_ws_bytes(desc(s_max=4096, sums=sums), 32, i) for i in range(1, 9)]
        assert n == sorted(n)
    # with sums, a row's scores of all positions come on top
    more = ld.ld_attn_decode_kv4_ws_bytes(desc(sums=P), 8, 1) - ld.ld_attn_decode_kv4_ws_bytes(desc(), 8, 1)
    assert more >= 2 * 8 * 4 * 100
    assert ld.ld_attn_decode_kv4_ws_bytes(kv, 8, 0) == ld.ld_attn_decode_kv4_ws_bytes(kv, 8, 9) == 0
    assert ld.ld_attn_decode_kv4_ws_bytes(kv, 7, 1) == 0


def test_binding_checks_tensors():
    n, m = ld.ld_kv4_code_bytes(desc()), ld.ld_kv4_scale_bytes(desc())
    u8 = lambda k: torch.zeros(k, dtype=torch.uint8)  # noqa: E731
    for codes, scales, sums, what in ((u8(n - 1), u8(m), None, "codes"), (torch.zeros(n, dtype=torch.int8), u8(m), None, "codes"),
                                      (u8(n), u8(m + 1), None, "scales"), (u8(n), torch.zeros(m), None, "scales"),
                                      (u8(n), u8(m), torch.zeros(2, 4, 99), "sums"),
                                      (u8(n), u8(m), torch.zeros(2, 4, 100, dtype=torch.float64), "sums"),
                                      (u8(n), u8(m), None, "device tensor")):
        with pytest.raises(ValueError, match=what):
            ld.kv4(codes, scales, sums=sums, **GOOD)
    rows = torch.zeros(2 * 3, (8 + 8) * 128, dtype=torch.bfloat16)
    for call in (store, attn):
        for kw in (dict(qkv=rows[:5]), dict(qkv=rows.float())):
            with pytest.raises(ValueError, match="qkv"):
                call(desc(), **kw)
        for sp in (torch.zeros(2, dtype=torch.int64), torch.zeros(3, dtype=torch.int32)):
            with pytest.raises(ValueError, match="seq_pos"):
                call(desc(), seq_pos=sp)
    with pytest.raises(ValueError, match="out"):
        load(desc(), out=torch.zeros(2, 3, 1023, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="o:"):
        attn(desc(), o=torch.zeros(2 * 3, 1023, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="idx"):
        evict(desc(sums=P), idx=torch.zeros(2, 4, 39, dtype=torch.int32))
    with pytest.raises(ValueError, match="idx"):
        evict(desc(sums=P), idx=torch.zeros(2, 4, 40, dtype=torch.int64))
    with pytest.raises(ValueError, match="seq_len"):
        evict(desc(sums=P), seq_len=torch.zeros(3, dtype=torch.int32))


def test_binding_refuses_another_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    rows = torch.zeros(2 * 3, (8 + 8) * 128, dtype=torch.bfloat16).as_subclass(OnDevice)
    for call in (store, attn):
        with pytest.raises(ValueError, match="current device"):
            call(desc(), qkv=rows)
    with pytest.raises(ValueError, match="current device"):
        evict(desc(sums=P), idx=torch.zeros(2, 4, 40, dtype=torch.int32).as_subclass(OnDevice))
    with pytest.raises(ValueError, match="current device"):
        attn(desc(), ws=torch.zeros(1 << 20, dtype=torch.uint8).as_subclass(OnDevice))
