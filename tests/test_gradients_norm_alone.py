"""The norm alone does not look at a tensor's output, whatever it is.  No GPU needed."""
import ctypes

import pytest

from paper_2605_08793_amd import binding as B
from test_experts_abi import NULL, P, WS, BIG, listed, tensor


@pytest.mark.parametrize("type", [0, 1, 2])
@pytest.mark.parametrize("out", [None, 0x1, 0x100003, 0x900001])
def test_any_output(out, type):
    size = ctypes.c_size_t()
    assert B.load().regot_grad_norm_workspace_bytes(1, listed(tensor(out=out, type=type)), ctypes.byref(size)) == 0 and size.value == 256
    # (refused for what is looked at behind the tensors)
    assert B.load().regot_grad_norm(1, listed(tensor(out=out, type=type)), None, WS, BIG, None) == NULL
    assert B.load().regot_grad_norm(1, listed(tensor(out=out, type=type)), P, None, 0, None) == NULL
