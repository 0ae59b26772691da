"""What the calls of 4-bit weights refuse, and their sizes (no GPU: no call here
reaches the HIP runtime)."""
import ctypes as C

import pytest
import torch

import paper_2609_05275_amd as ld
from tests.test_abi_kv8 import INVALID, SHAPE, UNSUPPORTED, WORKSPACE, OnDevice

P = 1 << 20
GOOD = dict(format=ld.LD_W4_INT4, group=64, n=48, k=200)


def desc(codes=P, scales=P, **kw):
    w = ld.ld_w4(**{**GOOD, **kw})
    w.codes, w.scales = codes, scales
    return w


def pack(w, src=P, rows=200):
    return ld._lib.ld_w4_pack(C.byref(w), src, rows, None)


def load(w, dst=P, rows=200):
    return ld._lib.ld_w4_load(C.byref(w), dst, rows, None)


def gemm(w, M=3, A=P, lda=200, g=None, eps=1e-5, Cm=P, ldc=48, alpha=1.0, R=None, ldr=48, act=0, ws=P, wsb=1 << 30):
    return ld._lib.ld_gemm_w4(M, A, lda, g, eps, C.byref(w), Cm, ldc, alpha, R, ldr, act, ws, wsb, None)


BAD_DESC = [(dict(format=2), INVALID), (dict(format=-1), INVALID), (dict(group=16), UNSUPPORTED),
            (dict(group=256), UNSUPPORTED), (dict(format=0, group=64), UNSUPPORTED), (dict(n=0), SHAPE), (dict(k=0), SHAPE),
            (dict(k=204), SHAPE), (dict(n=2 ** 30 + 1), SHAPE), (dict(k=2 ** 30 + 8), SHAPE),
            (dict(k=2 ** 29 + 8), SHAPE)]


@pytest.mark.parametrize("kw,code", BAD_DESC, ids=[str(k) for k, _ in BAD_DESC])
def test_descriptor_refused(kw, code):
    w = desc(**kw)
    assert ld.ld_w4_code_bytes(w) == 0 and ld.ld_w4_scale_bytes(w) == 0 and ld.ld_gemm_w4_ws_bytes(w, 1) == 0
    for call in (pack, load, gemm):
        assert call(w) == code and ld.last_error()


@pytest.mark.parametrize("kw", [dict(codes=None), dict(scales=None), dict(codes=P + 8), dict(scales=P + 4)], ids=str)
def test_buffers_refused(kw):
    for call in (pack, load, gemm):
        assert call(desc(**kw)) == INVALID


BAD_CALLS = [
    (pack, dict(src=None), INVALID), (pack, dict(src=P + 2), INVALID), (pack, dict(rows=192), SHAPE), (pack, dict(rows=204), SHAPE),
    (load, dict(dst=None), INVALID), (load, dict(dst=P + 2), INVALID), (load, dict(rows=192), SHAPE),
    (gemm, dict(M=0), SHAPE), (gemm, dict(M=65), SHAPE), (gemm, dict(act=3), INVALID), (gemm, dict(act=-1), INVALID),
    (gemm, dict(act=1, R=P), INVALID), (gemm, dict(act=2, R=P), INVALID), (gemm, dict(g=P, M=17), UNSUPPORTED),
    (gemm, dict(lda=192), SHAPE), (gemm, dict(lda=204), SHAPE), (gemm, dict(ldc=47), SHAPE), (gemm, dict(R=P, ldr=47), SHAPE),
    (gemm, dict(A=None), INVALID), (gemm, dict(Cm=None), INVALID), (gemm, dict(A=P + 2), INVALID), (gemm, dict(g=P + 2), INVALID),
    (gemm, dict(Cm=P + 1), INVALID), (gemm, dict(R=P + 1), INVALID), (gemm, dict(alpha=float("nan")), INVALID),
    (gemm, dict(g=P, eps=0.0), INVALID), (gemm, dict(A=P, Cm=P), INVALID),
]


@pytest.mark.parametrize("call,kw,code", BAD_CALLS, ids=[f"{c.__name__}-{k}" for c, k, _ in BAD_CALLS])
def test_call_refused(call, kw, code):
    assert call(desc(), **kw) == code and ld.last_error()


def test_swiglu_rows():
    assert gemm(desc(n=40), act=1) == SHAPE
    assert gemm(desc(n=47), act=1) == SHAPE


def test_workspace():
    w = desc(k=4000)
    n = ld.ld_gemm_w4_ws_bytes(w, 20)
    assert n > 0 and gemm(w, M=20, lda=4000, ws=None, Cm=2 * P) == WORKSPACE
    assert gemm(w, M=20, lda=4000, wsb=n - 1, Cm=2 * P) == WORKSPACE and gemm(w, M=20, lda=4000, ws=P + 8, Cm=2 * P) == INVALID
    assert ld.ld_gemm_w4_ws_bytes(w, 8) == ld.ld_gemm_w4_ws_bytes(desc(k=640), 64) == 0


def test_norm_of_long_rows():
    assert gemm(desc(k=8200), lda=8200, g=P) == UNSUPPORTED


def test_null_descriptor():
    lib, p = ld._lib, C.c_void_p(P)
    assert lib.ld_w4_code_bytes(None) == lib.ld_w4_scale_bytes(None) == lib.ld_gemm_w4_ws_bytes(None, 1, 0) == 0
    assert lib.ld_w4_pack(None, p, 8, None) == lib.ld_w4_load(None, p, 8, None) == INVALID
    assert lib.ld_gemm_w4(1, p, 8, None, 1e-5, None, p, 8, 1.0, None, 0, 0, None, 0, None) == INVALID


def test_sizes():
    for fmt, group, per in ((0, 32, 4), (1, 32, 8), (1, 64, 4), (1, 128, 2)):
        w = desc(format=fmt, group=group, n=47, k=264)
        assert ld.ld_w4_code_bytes(w) == 6 * 2 * 1024 and ld.ld_w4_scale_bytes(w) == 6 * 2 * 16 * per
    big = desc(n=2 ** 20, k=2 ** 20)                               # past 32 bits
    assert ld.ld_w4_code_bytes(big) == 2 ** 39
    for act in (0, 1, 2):
        n = [ld.ld_gemm_w4_ws_bytes(desc(), m, act) for m in range(1, 65)]
        assert n == sorted(n)
    assert ld.ld_gemm_w4_ws_bytes(desc(), 0) == ld.ld_gemm_w4_ws_bytes(desc(), 65) == ld.ld_gemm_w4_ws_bytes(desc(), 1, 3) == 0


def test_binding_checks_tensors():
    n, m = ld.ld_w4_code_bytes(desc()), ld.ld_w4_scale_bytes(desc())
    u8 = lambda k: torch.zeros(k, dtype=torch.uint8)  # noqa: E731
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    for codes, scales, what in ((u8(n + 1), bf(m // 2), "codes"), (u8(n), u8(m), "scales"), (u8(n), bf(m // 2 - 1), "scales"),
                                (u8(n), bf(m // 2), "device tensor")):
        with pytest.raises(ValueError, match=what):
            ld.w4(codes, scales, **GOOD)
    with pytest.raises(ValueError, match="scales"):
        ld.w4(u8(n), bf(m), format=0, group=32, n=48, k=200)
    w = desc()
    for call in (ld.ld_w4_pack, ld.ld_w4_load):
        for t in (bf(48, 192), bf(47, 200), torch.zeros(48, 200)):
            with pytest.raises(ValueError, match="expected bfloat16"):
                call(w, t, stream=0)


class Here(OnDevice):
    """A CPU tensor that says it lives on the first GPU."""
    device = torch.device("cuda", 0)

    def get_device(self):
        return 0


def test_binding_checks_the_projection(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    here = lambda *s: torch.zeros(*s, dtype=torch.bfloat16).as_subclass(Here)  # noqa: E731
    w = desc()
    good = dict(A=here(3, 200), C_out=here(3, 48))
    for bad, what in ((dict(A=here(3, 192)), "A:"), (dict(C_out=here(3, 47)), "C_out"), (dict(C_out=here(2, 48)), "C_out"),
                      (dict(R=here(3, 40)), "R:"), (dict(act=1), "C_out"), (dict(A=here(200, 3).t()), "last dimension"),
                      (dict(g=here(199)), "g:"), (dict(A=torch.zeros(3, 200).as_subclass(Here)), "A:"),
                      (dict(C_out=torch.zeros(3, 48, dtype=torch.bfloat16)), "current device")):
        with pytest.raises(ValueError, match=what):
            ld.ld_gemm_w4(w, **{**good, **bad}, stream=0)
    w.device = 1
    with pytest.raises(ValueError, match="current device"):
        ld.ld_gemm_w4(w, **good, stream=0)
