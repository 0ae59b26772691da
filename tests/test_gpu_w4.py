"""4-bit weights on the HIP path against the float64 oracle: codes and scales bit for
bit, projections within a bound that counts their roundings."""
import numpy as np
import pytest
import torch

import paper_2609_05275_amd as ld
from oracle import w4
from tests.gpu_util import DEV, f64

pytestmark = pytest.mark.gpu

KINDS = [(w4.E2M1, 32), (w4.INT4, 32), (w4.INT4, 64), (w4.INT4, 128)]
FORMATS = pytest.mark.parametrize("fmt,group", KINDS, ids=["e2m1", "int4_32", "int4_64", "int4_128"])


def device(fmt, group, n, k):
    probe = ld.w4(None, None, fmt, group, n, k)
    codes = torch.full((ld.ld_w4_code_bytes(probe),), 0xEE, dtype=torch.uint8, device=DEV)
    sb = ld.ld_w4_scale_bytes(probe)
    scales = torch.full((sb,), 0xFF, dtype=torch.uint8, device=DEV)
    return ld.w4(codes, scales if fmt == w4.E2M1 else scales.view(torch.bfloat16), fmt, group, n, k)


def packed(fmt, group, w):
    d = device(fmt, group, *w.shape)
    ld.ld_w4_pack(d, w.to(DEV))
    return d


def rand(rng, *shape, scale=1.0):
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(torch.bfloat16)


# ---------------------------------------------------------------- pack, load

@FORMATS
@pytest.mark.parametrize("n,k", [(1, 8), (7, 32), (8, 256), (9, 264), (24, 136), (33, 1000)])
def test_pack_and_load(fmt, group, n, k):
    rng = np.random.default_rng(n + k)
    w = rand(rng, n, k)
    w *= torch.from_numpy(2.0 ** rng.integers(-9, 9, (n, -(-k // 8)))).repeat_interleave(8, 1).to(torch.bfloat16)
    w[0, :8] = 0.0
    src = torch.full((n, k + 16), float("nan"), dtype=torch.bfloat16)     # rows apart, NaNs between
    src[:, :k] = w
    d = device(fmt, group, n, k)
    ld.ld_w4_pack(d, src.to(DEV)[:, :k])
    code, s = w4.quantise(fmt, group, f64(w))
    got = d.tensors[0].cpu().numpy().view(np.uint32).reshape(-(-n // 8), -(-k // 256), 64, 4)
    want = w4.dwords(fmt, code)
    if fmt == w4.E2M1:      # -0 is 0
        nib = lambda v: (v[..., None] >> np.arange(0, 32, 4, dtype=np.uint32)) & 15  # noqa: E731
        np.testing.assert_array_equal(np.where(nib(got) == 8, 0, nib(got)), np.where(nib(want) == 8, 0, nib(want)))
    else:
        np.testing.assert_array_equal(got, want)
    out = torch.full((n, k + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    ld.ld_w4_load(d, out[:, :k])
    v = (code * np.repeat(s, group, -1))[:, :k]
    np.testing.assert_array_equal(f64(out[:, :k]), w4.bf16(v))
    assert bool((out[:, k:] == 7.0).all())


@FORMATS
def test_pack_extreme_values(fmt, group):
    """Zeros, the smallest and largest scales, exact limits, infinities and NaNs."""
    w = torch.zeros(16, 256, dtype=torch.bfloat16)
    w[0, 0] = torch.finfo(torch.bfloat16).max
    w[1] = 2.0 ** -130
    w[2, 0], w[2, 1] = 6.0, 5.0
    w[3, 0], w[3, 1] = 6.03125, -2.5
    w[4, 0], w[4, 1:8] = 7.0, torch.arange(7) + 0.5
    w[5, 200] = float("inf")
    w[6, 100] = float("nan")
    w[7, 10] = -float("inf")
    w[8, 0] = 2.0 ** -99
    d = packed(fmt, group, w)
    out = torch.zeros(16, 256, dtype=torch.bfloat16, device=DEV)
    ld.ld_w4_load(d, out)
    with np.errstate(all="ignore"):
        v = w4.values(fmt, group, f64(w))
    want = np.where(np.isfinite(v), w4.bf16(np.where(np.isfinite(v), v, 0.0)), v)
    top = float(torch.finfo(torch.bfloat16).max)
    want = np.where(want > top, np.inf, want)           # 7 times a scale rounded up may pass the largest bf16
    np.testing.assert_array_equal(f64(out), want)
    assert np.isnan(want[5]).sum() == np.isnan(want[6]).sum() == np.isnan(want[7]).sum() == group


# --------------------------------------------------------------- projections

def bound(x, w, y, act, alpha, resid, K):
    """u = 2^-24.  Products are exact (4 bits by 8, or by 16 with a gain); a product
    of 32 k's adds up to 32 terms, the sums over K / 32 of those, groups, waves and halves
    follow, each addition within 2 u of the magnitudes' sum; the scales, alpha and 1/rms
    (a sum of K squares, a division, a square root) some u more.  y: the exact
    result before the activation.  Then the activation's, and half a bf16 step."""
    u = 2.0 ** -24
    mag = abs(alpha) * (np.abs(x) @ np.abs(w).T)
    e = u * (2 * (32 + K / 32 + 32) + 2 * (K / 32 + 40) + 16) * mag
    if act == "swiglu":
        (a, b), (ea, eb) = np.split(y, 2, -1), np.split(e, 2, -1)
        s = 1 / (1 + np.exp(-a))
        out = a * s * b
        e = 1.1 * ea * (np.abs(b) + eb) + np.abs(a * s) * eb + u * (12 + 4 * np.abs(a)) * np.abs(out)
    elif act == "relu2":
        out = np.maximum(y, 0) ** 2
        e = 2 * np.maximum(y, 0) * e + e * e + u * out
    else:
        out = y if resid is None else y + resid
        e = e + u * np.abs(out)
    return out, 1.01 * e + 2.0 ** -8 * np.abs(out) + 1e-38


def run(fmt, group, M, N, K, act="none", norm=False, resid=False, alpha=1.0, seed=0, scale=0.05, extra=0, inplace=False):
    rng = np.random.default_rng(seed + M + N + K)
    rows = 2 * N if act == "swiglu" else N
    w = rand(rng, rows, K, scale=scale)
    d = packed(fmt, group, w)
    wv = w4.values(fmt, group, f64(w))
    # rows apart, with NaNs between them
    x = torch.full((M, K + 8 * extra), float("nan"), dtype=torch.bfloat16)
    x[:, :K] = rand(rng, M, K)
    g = (1 + rand(rng, K, scale=0.2)) if norm else None
    R = rand(rng, M, N) if resid else None
    c = torch.full((M, N + 3 * extra), 7.0, dtype=torch.bfloat16, device=DEV)
    if inplace:
        c[:, :N] = R.to(DEV)
    ws = torch.full((ld.ld_gemm_w4_ws_bytes(d, M, {"none": 0, "swiglu": 1, "relu2": 2}[act]),), 0xFF, dtype=torch.uint8, device=DEV)
    xd, gd, rd = x.to(DEV), None if g is None else g.to(DEV), None if R is None else R.to(DEV)
    out = []
    for _ in range(2):
        if inplace:
            c[:, :N] = rd
        ld.ld_gemm_w4(d, xd[:, :K], c[:, :N], ws, g=gd, eps=1e-5, alpha=alpha, R=c[:, :N] if inplace else rd,
                      act={"none": 0, "swiglu": 1, "relu2": 2}[act])
        out.append(c.clone())
    assert torch.equal(out[0], out[1])
    assert bool((c[:, N:] == 7.0).all())
    x64 = f64(x[:, :K])
    if norm:
        x64 = x64 / np.sqrt(np.mean(x64 ** 2, -1, keepdims=True) + 1e-5) * f64(g)
    y = alpha * (x64 @ wv.T)
    want, e = bound(x64, wv, y, act, alpha, None if R is None else f64(R), K)
    np.testing.assert_allclose(want, w4.project(x64, wv, alpha=alpha, R=None if R is None else f64(R), act=act), rtol=1e-12, atol=1e-300)
    far = np.abs(f64(c[:, :N]) - want) / e
    assert np.max(far) <= 1.0, (np.max(far), np.unravel_index(np.argmax(far), far.shape))


@FORMATS
@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16, 17, 31, 33, 48, 64])
@pytest.mark.parametrize("N,K", [(40, 256), (17, 1032)])
def test_rows(fmt, group, M, N, K):
    run(fmt, group, M, N, K, resid=M % 2 == 0, alpha=0.5 if M % 3 else 1.0, extra=M % 2)


@FORMATS
@pytest.mark.parametrize("K", [8, 24, 32, 40, 120, 128, 136, 248, 256, 512, 520, 768, 2048, 2056, 4096, 4104, 5504, 8192, 8200,
                               11008, 16384, 16392, 20000])
def test_k(fmt, group, K):
    """One row and several, with and without a norm where there can be one."""
    run(fmt, group, 1, 24, K, norm=K <= 8192)
    run(fmt, group, 5, 16, K, act="swiglu", norm=K <= 8192)
    run(fmt, group, 12, 9, K, norm=K <= 8192 and K % 16 == 8, resid=True)


@FORMATS
@pytest.mark.parametrize("N", [1, 7, 8, 9, 63, 1000, 2048, 2053, 6001, 20000])
@pytest.mark.parametrize("M", [1, 6, 40])
def test_n(fmt, group, N, M):
    run(fmt, group, M, N, 256 if N > 2500 else 520, act="relu2" if N % 2 else "none")


@FORMATS
@pytest.mark.parametrize("M", [1, 8, 16])
@pytest.mark.parametrize("act", ["none", "swiglu", "relu2"])
def test_norm(fmt, group, M, act):
    run(fmt, group, M, 504, 768, act=act, norm=True, alpha=1.5, extra=1)


@pytest.mark.parametrize("M,N,K,act", [(1, 5504, 2048, "swiglu"), (8, 2304, 768, "none"), (3, 11008, 4096, "swiglu"),
                                       (48, 11008, 4096, "swiglu"), (64, 2048, 5504, "none"), (20, 16384, 2048, "relu2"),
                                       (1, 40000, 4096, "none")])
@pytest.mark.parametrize("fmt,group", [(w4.E2M1, 32), (w4.INT4, 128)], ids=["e2m1", "int4_128"])
def test_layer_shapes(fmt, group, M, N, K, act):
    run(fmt, group, M, N, K, act=act, norm=M <= 16)


@FORMATS
@pytest.mark.parametrize("M", [17, 33, 49, 64])
@pytest.mark.parametrize("K", [640, 648, 848, 856, 1272, 1288, 2568, 4104])
def test_rows_as_they_lie_and_laid_out(fmt, group, M, K):
    """Both sides of where rows are laid out first, the last chunk a part of one."""
    run(fmt, group, M, 41, K, resid=True, extra=1)
    run(fmt, group, M, 32, K, act="swiglu")


@pytest.mark.parametrize("fmt,group", [(w4.E2M1, 32), (w4.INT4, 64)], ids=["e2m1", "int4_64"])
@pytest.mark.parametrize("M,N,K", [(20, 4105, 2568), (40, 4105, 1032), (40, 8209, 1032), (60, 16401, 776), (64, 4121, 264), (33, 16401, 264),
                                   (12, 16393, 520), (12, 16393, 2568)])
def test_columns_of_laid_out_rows(fmt, group, M, N, K):
    """One to six groups of columns a workgroup, the last workgroup's partly behind N."""
    run(fmt, group, M, N, K, act="relu2" if M == 60 else "none")


def test_in_place_residual():
    for M in (1, 9, 50):
        run(w4.INT4, 64, M, 72, 512, resid=True, alpha=0.7, inplace=True)


@FORMATS
def test_nan_and_infinite(fmt, group):
    """A NaN group of weights makes its column NaN, a NaN or infinite input its row; no
    others."""
    rng = np.random.default_rng(3)
    w, x = rand(rng, 21, 600), rand(rng, 11, 600)
    clean = packed(fmt, group, w)
    w[5, 300] = float("nan")
    bad = packed(fmt, group, w)
    out = torch.zeros(2, 11, 21, dtype=torch.bfloat16, device=DEV)
    ws = torch.zeros(ld.ld_gemm_w4_ws_bytes(clean, 11), dtype=torch.uint8, device=DEV)
    ld.ld_gemm_w4(clean, x.to(DEV), out[0], ws)
    ld.ld_gemm_w4(bad, x.to(DEV), out[1], ws)
    assert bool(torch.isnan(out[1][:, 5]).all())
    keep = [i for i in range(21) if i != 5]
    assert torch.equal(out[0][:, keep], out[1][:, keep])
    y = x.clone()
    y[2, 7], y[9, 599] = float("nan"), float("inf")
    ld.ld_gemm_w4(clean, y.to(DEV), out[1], ws)
    assert not bool(torch.isfinite(out[1][[2, 9]]).any())
    keep = [i for i in range(11) if i not in (2, 9)]
    assert torch.equal(out[0][keep], out[1][keep])


def test_weights_that_cancel():
    """Rows whose sums are a small rest of large terms: what a rounded scale or sum of
    a group would leave shows."""
    K = 4096
    rng = np.random.default_rng(0)
    w = rand(rng, 8, K)
    w[:, 1::2] = -w[:, 0::2]
    w[0, 4] += 0.5
    for fmt, group in KINDS:
        d = packed(fmt, group, w)
        wv = w4.values(fmt, group, f64(w))
        x = torch.ones(2, K, dtype=torch.bfloat16)
        out = torch.zeros(2, 8, dtype=torch.bfloat16, device=DEV)
        ld.ld_gemm_w4(d, x.to(DEV), out)
        want, e = bound(f64(x), wv, f64(x) @ wv.T, "none", 1.0, None, K)
        assert np.all(np.abs(f64(out) - want) <= e)


def test_captured_and_on_another_stream():
    rng = np.random.default_rng(1)
    d = packed(w4.E2M1, 32, rand(rng, 2 * 264, 2048, scale=0.02))
    x = rand(rng, 4, 2048).to(DEV)
    g = (1 + rand(rng, 2048, scale=0.1)).to(DEV)
    ws = torch.zeros(ld.ld_gemm_w4_ws_bytes(d, 64, 1), dtype=torch.uint8, device=DEV)
    out, cap = (torch.zeros(4, 264, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    call = lambda c: ld.ld_gemm_w4(d, x, c, ws, g=g, act=ld.DEC_ACT_SWIGLU)  # noqa: E731
    call(cap)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call(cap)
    for i in range(3):
        x.copy_(rand(rng, 4, 2048))
        call(out)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, cap)
    with torch.cuda.stream(s):
        cap.zero_()
        call(cap)
    torch.cuda.synchronize()
    assert torch.equal(out, cap)


def test_codes_past_32_bits():
    """Weights of more than 2^32 bytes of codes: the last rows' columns."""
    N, K = 540000, 16384
    d = device(w4.E2M1, 32, N, K)
    assert d.tensors[0].numel() > 2 ** 32
    d.tensors[0].zero_()
    d.tensors[1].fill_(127)
    rng = np.random.default_rng(0)
    w = rand(rng, 16, K)
    small = packed(w4.E2M1, 32, w)
    nb, sb = small.tensors[0].numel(), small.tensors[1].numel()
    d.tensors[0][-nb:] = small.tensors[0]
    d.tensors[1][-sb:] = small.tensors[1]
    x = rand(rng, 2, K).to(DEV)
    out, want = torch.zeros(2, N, dtype=torch.bfloat16, device=DEV), torch.zeros(2, 16, dtype=torch.bfloat16, device=DEV)
    ld.ld_gemm_w4(d, x, out, torch.zeros(max(1, ld.ld_gemm_w4_ws_bytes(d, 2)), dtype=torch.uint8, device=DEV))
    ld.ld_gemm_w4(small, x, want, torch.zeros(max(1, ld.ld_gemm_w4_ws_bytes(small, 2)), dtype=torch.uint8, device=DEV))
    assert not bool(out[:, :-16].any())
    # (more tiles may be taken by another variant: the same sums in another order)
    e = bound(f64(x), w4.values(w4.E2M1, 32, f64(w)), f64(want), "none", 1.0, None, K)[1]
    assert np.all(np.abs(f64(out[:, -16:]) - f64(want)) <= 2 * e)


def test_many_rows_by_codes_past_32_bits():
    """The same with rows that are laid out: tiles of the last workgroups, and the last of all
    alone."""
    N, K, M = 540008, 16384, 20
    d = device(w4.E2M1, 32, N, K)
    d.tensors[0].zero_()
    d.tensors[1].fill_(127)
    rng = np.random.default_rng(2)
    w = rand(rng, 24, K)
    small = packed(w4.E2M1, 32, w)
    d.tensors[0][-small.tensors[0].numel():] = small.tensors[0]
    d.tensors[1][-small.tensors[1].numel():] = small.tensors[1]
    x = rand(rng, M, K).to(DEV)
    out, want = torch.zeros(M, N, dtype=torch.bfloat16, device=DEV), torch.zeros(M, 24, dtype=torch.bfloat16, device=DEV)
    ws = torch.zeros(ld.ld_gemm_w4_ws_bytes(d, M), dtype=torch.uint8, device=DEV)
    ld.ld_gemm_w4(d, x, out, ws)
    ld.ld_gemm_w4(small, x, want, ws)
    assert not bool(out[:, :-24].any())
    e = bound(f64(x), w4.values(w4.E2M1, 32, f64(w)), f64(want), "none", 1.0, None, K)[1]
    assert np.all(np.abs(f64(out[:, -24:]) - f64(want)) <= 2 * e)


def test_two_captured_calls_share_a_workspace():
    """What a call lays out in its workspace is its own rows, replay after replay."""
    rng = np.random.default_rng(4)
    ds = [packed(w4.INT4, 64, rand(rng, 200, K, scale=0.02)) for K in (776, 2048)]
    xs = [rand(rng, M, K).to(DEV) for M, K in ((40, 776), (20, 2048))]
    ws = torch.zeros(max(ld.ld_gemm_w4_ws_bytes(d, 64) for d in ds), dtype=torch.uint8, device=DEV)
    cap, out = ([torch.zeros(x.shape[0], 200, dtype=torch.bfloat16, device=DEV) for x in xs] for _ in range(2))
    graphs = []
    for d, x, c in zip(ds, xs, cap):
        ld.ld_gemm_w4(d, x, c, ws)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            ld.ld_gemm_w4(d, x, c, ws)
    for i in range(3):
        for x in xs:
            x.copy_(rand(rng, *x.shape))
        for g in graphs if i % 2 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        for d, x, o, c in zip(ds, xs, out, cap):
            ld.ld_gemm_w4(d, x, o, ws)
            assert torch.equal(o, c)
