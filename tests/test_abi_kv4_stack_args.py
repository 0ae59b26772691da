"""Rows, scratch and gains that the stack calls over 4-bit caches and weights refuse
(no GPU: nothing here reaches the HIP runtime)."""
import pytest

import paper_2609_05275_amd as ld
from tests.test_abi_kv4_stack import CALLS, P
from tests.test_abi_kv8 import INVALID, Raw


@pytest.mark.parametrize("off", [2, 8])
def test_alignment(off):
    for call in CALLS:
        for kw in (dict(x=P + off), dict(ws=Raw(P + off))):
            with pytest.raises(ld.LdError, match="16-byte aligned") as e:
                call(**kw)
            assert e.value.status == INVALID
