"""Projections by 4-bit weights that keep their rows in registers take no workspace,
and give what they give with one."""
import numpy as np
import pytest
import torch

import paper_2609_05275_amd as ld
from tests.gpu_util import DEV
from tests.test_gpu_w4 import FORMATS, packed, rand

pytestmark = pytest.mark.gpu


@FORMATS
@pytest.mark.parametrize("M", [9, 16])
@pytest.mark.parametrize("N,K,norm", [(40, 1288, False), (40, 4096, False), (40, 4104, True), (16, 8192, True), (16400, 1288, True)])
def test_without_a_workspace(fmt, group, M, N, K, norm):
    rng = np.random.default_rng(M + N + K)
    d, x = packed(fmt, group, rand(rng, N, K, scale=0.05)), rand(rng, M, K).to(DEV)
    g = (1 + rand(rng, K, scale=0.1)).to(DEV) if norm else None
    ws = torch.full((M * K * 8 + 4096,), 0xFF, dtype=torch.uint8, device=DEV)
    a, b = (torch.zeros(M, N, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ld.ld_gemm_w4(d, x, a, ws, g=g)
    ld.ld_gemm_w4(d, x, b, None, g=g)
    assert torch.equal(a, b) and bool(a.any()) and bool((ws == 0xFF).all())
