"""Which projections by 4-bit weights ask for a workspace: those whose rows are laid out
in it (no GPU: no call here reaches the HIP runtime)."""
import pytest

import paper_2609_05275_amd as ld
from tests.test_abi_kv8 import WORKSPACE
from tests.test_abi_w4 import P, desc, gemm


@pytest.mark.parametrize("n,k,M,some", [
    (48, 2048, 8, False), (48, 16384, 8, False),                     # up to 8 rows none
    (48, 2048, 9, False), (48, 4096, 16, False), (16384, 4096, 16, False),   # held in registers
    (48, 4104, 9, True), (16385, 2048, 16, True), (16392, 1288, 9, True),
    (16392, 1280, 16, False),                                        # read where they lie
    (48, 1280, 17, False), (48, 1288, 17, True), (48, 640, 64, False), (48, 648, 64, True)])
def test_sizes(n, k, M, some):
    w = desc(n=n, k=k)
    size = ld.ld_gemm_w4_ws_bytes(w, M)
    assert size == ((M + 15) // 16 * 16 * ((k + 255) // 256 * 256) * 2 if some else 0)
    assert all(ld.ld_gemm_w4_ws_bytes(w, m) <= size for m in range(1, M))
    if some:
        assert gemm(w, M=M, lda=k, ldc=n, Cm=2 * P, ws=None) == WORKSPACE
        assert gemm(w, M=M, lda=k, ldc=n, Cm=2 * P, wsb=size - 1) == WORKSPACE


def test_a_step_has_scratch_for_every_projection():
    """Rows of a stack's step beyond 64 go 64 at a time, the rest too."""
    for B, d, f in ((1, 256, 512), (9, 256, 5504), (9, 4096, 11008), (20, 2048, 5504), (72, 1024, 8192), (80, 256, 16384)):
        c = ld.config(batch=B, seq=64, d_model=d, n_heads=d // 128, d_ff=f, dtype=ld.LD_BF16)
        size = ld.ld_decode_kv4_ws_bytes(c, 1, 100)
        for rows in {min(B, 64), B % 64} - {0}:
            for n, k in ((3 * d, d), (d, d), (2 * f, d), (d, f)):
                assert ld.ld_gemm_w4_ws_bytes(desc(n=n, k=k), rows) < size
