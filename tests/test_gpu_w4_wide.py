"""Projections by 4-bit weights of so many rows that their workgroups go in several
launches: the last columns are right and none is left out."""
import numpy as np
import pytest
import torch

import paper_2609_05275_amd as ld
from oracle import w4
from tests.gpu_util import DEV, f64
from tests.test_gpu_w4 import bound, device, packed, rand

pytestmark = pytest.mark.gpu


def last_columns(N, K, M, act="none", norm=False, last=24):
    """The last rows of W (SwiGLU: of both halves) are random, the others zeros: their columns
    against float64, the others' all zero."""
    rng = np.random.default_rng(N + K + M)
    code = {"none": 0, "swiglu": 1, "relu2": 2}[act]
    halves = 2 if act == "swiglu" else 1
    d = device(w4.E2M1, 32, halves * N, K)
    d.tensors[0].zero_()
    d.tensors[1].fill_(127)
    wv = []
    for h in range(halves):
        w = rand(rng, last, K, scale=0.2)
        small = packed(w4.E2M1, 32, w)
        for to, t in zip(d.tensors, small.tensors):
            end = to.numel() // halves * (h + 1)
            to[end - t.numel():end] = t
        wv.append(w4.values(w4.E2M1, 32, f64(w)))
    x = rand(rng, M, K)
    g = 1 + rand(rng, K, scale=0.1) if norm else None
    out = torch.full((M, N), 7.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(ld.ld_gemm_w4_ws_bytes(d, M, code), dtype=torch.uint8, device=DEV)
    ld.ld_gemm_w4(d, x.to(DEV), out, ws, g=None if g is None else g.to(DEV), act=code)
    for m in range(M):      # (a row at a time: less memory)
        assert not bool(out[m, :-last].any()), m
    x64 = f64(x)
    if norm:
        x64 = x64 / np.sqrt(np.mean(x64 ** 2, -1, keepdims=True) + 1e-5) * f64(g)
    wv = np.concatenate(wv)
    want, e = bound(x64, wv, x64 @ wv.T, act, 1.0, None, K)
    assert np.max(np.abs(f64(out[:, -last:]) - want) / e) <= 1.0
    del d, out, ws
    torch.cuda.empty_cache()


@pytest.mark.parametrize("N,K,M,act,norm", [
    (1080008, 4104, 12, "none", True),          # rows and codes beside each other, 8 columns a workgroup
    (1080008, 4104, 9, "swiglu", True),
    (4400008, 264, 12, "none", False),          # rows where they lie, 32 columns a workgroup
    (2200008, 1032, 30, "swiglu", False),       # 16 columns of both halves
    (4400008, 1304, 20, "none", False),         # laid out
    (12600008, 1032, 33, "relu2", False),       # 96 columns a workgroup
], ids=["long", "long_swiglu", "as_they_lie", "as_they_lie_swiglu", "laid_out", "laid_out_48"])
def test_several_launches(N, K, M, act, norm):
    last_columns(N, K, M, act, norm)


def test_past_32_bits_of_threads():
    """2^28 columns, 32 a workgroup of 512 threads: more than the 2^32 threads of one launch; 34 GB of
    codes."""
    if torch.cuda.mem_get_info()[0] < 64 << 30:
        pytest.skip("needs 64 GB")
    last_columns(2 ** 28 + 24, 8, 12)
