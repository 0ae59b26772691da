"""What the 8-bit cache's calls refuse, and its sizes (no GPU: no call here
reaches the HIP runtime)."""
import ctypes as C

import pytest
import torch

import paper_2609_05275_amd as ld

GOOD = dict(format=ld.LD_KV8_E4M3, block=64, n_seq=2, n_kv_heads=4, d_head=128, s_max=100)
INVALID, SHAPE, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4


class Raw:
    """An address that is never followed."""

    def __init__(self, addr, n=1 << 40):
        self.addr, self.n = addr, n

    def data_ptr(self):
        return self.addr

    def numel(self):
        return self.n

    def element_size(self):
        return 1


A = Raw(1 << 20)


def desc(codes=1 << 20, scales=1 << 20, **kw):
    kv = ld.ld_kv8(**{**GOOD, **kw})
    kv.codes, kv.scales = codes, scales
    return kv


def store(kv, n_heads=8, n_new=3, pos=5, qkv=A, seq_pos=None):
    ld.ld_kv8_store(kv, n_heads, n_new, pos, qkv, seq_pos=seq_pos, stream=0)


def load(kv, pos=5, n=3, out=A, seq_len=None):
    ld.ld_kv8_load(kv, pos, n, out, seq_len=seq_len, stream=0)


def attn(kv, n_heads=8, pos=5, n_new=3, qkv=A, o=A, ws=A, seq_pos=None, alibi=0):
    ld.ld_attn_decode_kv8(kv, n_heads, pos, n_new, qkv, o, ws, seq_pos=seq_pos, alibi=alibi, stream=0)


BAD_DESC = [(dict(format=2), INVALID), (dict(format=-1), INVALID), (dict(block=8), UNSUPPORTED),
            (dict(block=48), UNSUPPORTED), (dict(block=256), UNSUPPORTED), (dict(block=0), UNSUPPORTED),
            (dict(d_head=96), UNSUPPORTED), (dict(d_head=256), UNSUPPORTED), (dict(n_seq=0), SHAPE),
            (dict(n_kv_heads=0), SHAPE), (dict(s_max=0), SHAPE), (dict(n_seq=65536), SHAPE),
            (dict(n_kv_heads=32768), SHAPE), (dict(s_max=2 ** 31 - 1), SHAPE),
            (dict(n_seq=1, n_kv_heads=1, s_max=2 ** 30 + 1), SHAPE),
            (dict(n_seq=60000, n_kv_heads=30000), SHAPE)]


@pytest.mark.parametrize("kw,code", BAD_DESC, ids=[str(k) for k, _ in BAD_DESC])
def test_descriptor_refused(kw, code):
    kv = desc(**kw)
    assert ld.ld_kv8_code_bytes(kv) == 0 and ld.ld_kv8_scale_bytes(kv) == 0
    assert ld.ld_attn_decode_kv8_ws_bytes(kv, 8, 1) == 0
    for call in (store, load, attn):
        with pytest.raises(ld.LdError) as e:
            call(kv)
        assert e.value.status == code


BAD_BUFFERS = [dict(codes=None), dict(scales=None), dict(codes=(1 << 20) + 8), dict(scales=(1 << 20) + 2)]


@pytest.mark.parametrize("kw", BAD_BUFFERS, ids=[str(k) for k in BAD_BUFFERS])
def test_buffers_refused(kw):
    for call in (store, load, attn):
        with pytest.raises(ld.LdError) as e:
            call(desc(**kw))
        assert e.value.status == INVALID


OFF, NULL = Raw((1 << 20) + 8), None
BAD_CALLS = [
    (store, dict(n_heads=6), SHAPE), (store, dict(n_heads=0), SHAPE), (store, dict(n_heads=65536), SHAPE),
    (store, dict(n_new=0), SHAPE), (store, dict(pos=-1), SHAPE), (store, dict(pos=98), SHAPE),
    (store, dict(pos=2 ** 31 - 1), SHAPE), (store, dict(qkv=NULL), INVALID), (store, dict(qkv=OFF), INVALID),
    (store, dict(seq_pos=Raw((1 << 20) + 2)), INVALID),
    (load, dict(n=0), SHAPE), (load, dict(pos=-1), SHAPE), (load, dict(pos=98), SHAPE), (load, dict(out=NULL), INVALID),
    (load, dict(out=OFF), INVALID), (load, dict(seq_len=Raw((1 << 20) + 2)), INVALID),
    (attn, dict(n_heads=6), SHAPE), (attn, dict(n_new=0), INVALID), (attn, dict(n_new=9), INVALID),
    (attn, dict(alibi=2), INVALID), (attn, dict(pos=-1), SHAPE), (attn, dict(pos=98), SHAPE),
    (attn, dict(qkv=NULL), INVALID), (attn, dict(o=NULL), INVALID), (attn, dict(qkv=OFF), INVALID),
    (attn, dict(ws=Raw((1 << 20) + 4)), INVALID), (attn, dict(ws=Raw(1 << 20, 64)), WORKSPACE),
    (attn, dict(seq_pos=Raw((1 << 20) + 1)), INVALID),
]


@pytest.mark.parametrize("call,kw,code", BAD_CALLS, ids=[f"{c.__name__}-{next(iter(k))}-{i}" for i, (c, k, _) in enumerate(BAD_CALLS)])
def test_call_refused(call, kw, code):
    with pytest.raises(ld.LdError) as e:
        call(desc(), **kw)
    assert e.value.status == code and ld.last_error()


def test_null_descriptor():
    lib = ld._lib
    assert lib.ld_kv8_code_bytes(None) == 0
    assert lib.ld_kv8_store(None, 8, 1, 0, None, C.c_void_p(1 << 20), None) == INVALID
    assert lib.ld_kv8_load(None, 0, 1, None, C.c_void_p(1 << 20), None) == INVALID
    p = C.c_void_p(1 << 20)
    assert lib.ld_attn_decode_kv8(None, 8, 0, 0, None, 1, p, p, p, 1 << 30, None) == INVALID


def test_sizes():
    kv = desc()
    assert ld.ld_kv8_code_bytes(kv) == 2 * 4 * 2 * 112 * 128       # 100 positions in 112
    assert ld.ld_kv8_scale_bytes(kv) == 2 * 4 * 2 * 2 * 4
    big = desc(n_seq=64, n_kv_heads=32, s_max=131072)              # past 32 bits
    assert ld.ld_kv8_code_bytes(big) == 64 * 32 * 2 * 131072 * 128
    # the workspace of a cache holds what any shorter one needs
    last = 0
    for s_max in (1, 64, 65, 256, 300, 1000, 4096, 70000, 131072):
        n = ld.ld_attn_decode_kv8_ws_bytes(desc(n_seq=1, s_max=s_max), 8, 3)
        assert n >= last > -1
        last = n
    assert ld.ld_attn_decode_kv8_ws_bytes(kv, 8, 0) == ld.ld_attn_decode_kv8_ws_bytes(kv, 8, 9) == 0
    assert ld.ld_attn_decode_kv8_ws_bytes(kv, 7, 1) == 0


def test_binding_checks_tensors():
    n = ld.ld_kv8_code_bytes(desc())
    with pytest.raises(ValueError, match="codes"):
        ld.kv8(torch.zeros(n - 1, dtype=torch.uint8), None, **GOOD)
    with pytest.raises(ValueError, match="codes"):
        ld.kv8(torch.zeros(n, dtype=torch.int8), None, **GOOD)
    with pytest.raises(ValueError, match="scales"):
        ld.kv8(torch.zeros(n, dtype=torch.uint8), torch.zeros(31), **GOOD)
    with pytest.raises(ValueError, match="device tensor"):
        ld.kv8(torch.zeros(n, dtype=torch.uint8), torch.zeros(32), **GOOD)
    rows = torch.zeros(2 * 3, (8 + 8) * 128, dtype=torch.bfloat16)
    for call in (store, attn):
        with pytest.raises(ValueError, match="qkv"):
            call(desc(), qkv=rows[:5])
        with pytest.raises(ValueError, match="qkv"):
            call(desc(), qkv=rows.float())
        with pytest.raises(ValueError, match="seq_pos"):
            call(desc(), qkv=A, seq_pos=torch.zeros(2, dtype=torch.int64))
        with pytest.raises(ValueError, match="seq_pos"):
            call(desc(), qkv=A, seq_pos=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="out"):
        load(desc(), out=torch.zeros(2, 3, 1023, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="o:"):
        attn(desc(), o=torch.zeros(2 * 3, 1023, dtype=torch.bfloat16))


class OnDevice(torch.Tensor):
    """A CPU tensor that says it lives on another GPU."""
    is_cuda = True
    device = torch.device("cuda", 1)


def test_binding_refuses_another_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    rows = torch.zeros(2 * 3, (8 + 8) * 128, dtype=torch.bfloat16).as_subclass(OnDevice)
    for call in (store, attn):
        with pytest.raises(ValueError, match="current device"):
            call(desc(), qkv=rows)
    with pytest.raises(ValueError, match="current device"):
        load(desc(), out=torch.zeros(2, 3, 1024, dtype=torch.bfloat16).as_subclass(OnDevice))
