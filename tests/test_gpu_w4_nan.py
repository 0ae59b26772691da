"""A NaN reaches the output of every projection by 4-bit weights, through each
activation."""
import numpy as np
import pytest
import torch

import paper_2609_05275_amd as ld
from oracle import w4
from tests.gpu_util import DEV
from tests.test_gpu_w4 import FORMATS, packed, rand

pytestmark = pytest.mark.gpu


@FORMATS
@pytest.mark.parametrize("act", ["none", "swiglu", "relu2"])
@pytest.mark.parametrize("M,K,norm", [(3, 520, True), (3, 20000, False), (12, 520, False), (12, 5504, True), (40, 520, False),
                                      (40, 2056, False)],
                         ids=["held", "long", "held_16", "long_norm", "as_they_lie", "laid_out"])
def test_nan_passes_the_activation(fmt, group, act, M, K, norm):
    """A NaN weight makes its column NaN (SwiGLU: be it the gate's or the up's), a NaN input
    its row; the others stay as they were."""
    rng = np.random.default_rng(M + K)
    N, code = 24, {"none": 0, "swiglu": 1, "relu2": 2}[act]
    w, x = rand(rng, N * (2 if act == "swiglu" else 1), K, scale=0.05), rand(rng, M, K)
    g = (1 + rand(rng, K, scale=0.1)).to(DEV) if norm else None
    clean = packed(fmt, group, w)
    w[5, K - 1] = float("nan")
    if act == "swiglu":
        w[N + 9, 3] = float("nan")
    bad = packed(fmt, group, w)
    ws = torch.zeros(ld.ld_gemm_w4_ws_bytes(clean, M, code), dtype=torch.uint8, device=DEV)
    out = torch.zeros(3, M, N, dtype=torch.bfloat16, device=DEV)
    y = x.clone()
    y[2, 7] = float("nan")
    for o, d, a in zip(out, (clean, bad, clean), (x, x, y)):
        ld.ld_gemm_w4(d, a.to(DEV), o, ws, g=g, act=code)
    nan = torch.zeros(2, M, N, dtype=torch.bool)
    nan[0][:, [5, 9] if act == "swiglu" else [5]] = True
    nan[1][2] = True
    assert bool(torch.isfinite(out[0]).all())
    for o, m in zip(out[1:].cpu(), nan):
        assert torch.equal(torch.isnan(o), m)
        assert torch.equal(o[~m], out[0].cpu()[~m])
