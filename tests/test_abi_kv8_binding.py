"""What the binding of the stack calls over 8-bit caches refuses in the tensors it
is given (no GPU: nothing here reaches the HIP runtime)."""
import pytest
import torch

from tests.test_abi_kv8 import OnDevice
from tests.test_abi_kv8_stack import decode, evaluate

ROWS = 2 * 64 * 256     # x of ld_stack_eval_kv8 in these tests' configuration


@pytest.mark.parametrize("x", [torch.zeros(ROWS - 1, dtype=torch.bfloat16), torch.zeros(ROWS + 256, dtype=torch.bfloat16),
                               torch.zeros(ROWS), torch.zeros(ROWS, dtype=torch.float16)],
                         ids=["short", "long", "float32", "float16"])
def test_eval_checks_x(x):
    with pytest.raises(ValueError, match="x: (dtype|[0-9]+ elements)"):
        evaluate(x=x)


def elsewhere(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)


def test_another_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    ws = elsewhere(1 << 16, dtype=torch.uint8)
    for call, x in ((evaluate, elsewhere(2, 64, 256)), (decode, elsewhere(2, 1, 256))):
        with pytest.raises(ValueError, match="x: .*current device"):
            call(x=x)
        with pytest.raises(ValueError, match="ws: .*current device"):
            call(ws=ws)
    with pytest.raises(ValueError, match="seq_pos: .*current device"):
        decode(seq_pos=elsewhere(2, dtype=torch.int32))
