"""The counter records that bench.py reports beside its times are of the sources
as they are: it leaves out those of kernels whose sources have changed since, so
a change to them wants the records measured again."""
import os

import pytest

from paper_2609_05275_amd import profsum

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def current(rec):
    return profsum.source_hash(rec["source"], ROOT) == rec["source_sha256"]


@pytest.mark.parametrize("workload", ["1b", "paper_3p9b"])
def test_traffic(workload):
    rec = profsum.read_traffic(os.path.join(ROOT, "profiles", f"ld_gemm_bf16_tn_nn_256_{workload}_traffic.md"))
    assert rec["source"] == profsum.kernel_source("ld_gemm_bf16_tn_nn_256") and current(rec)


@pytest.mark.parametrize("workload", ["1b", "125m"])
def test_counters(workload):
    recs = profsum.read_counters(os.path.join(ROOT, "profiles", f"stack_step_{workload}_counters.md"))
    recs = {k: r for k, r in recs.items() if r.get("source")}
    assert {k.split("<")[0] for k in recs} > {"ld_gemm_bf16_nt_256", "ld_attn_fwd_bf16", "ld_rmsnorm_fwd_k"}
    assert [k for k, r in recs.items() if not current(r)] == []
