"""Gradients that a program replaces by tensors of its own: those that no call would write are refused, whatever has been called before.  No GPU needed."""
import pytest
import torch

from paper_2605_08793_amd.experts import ExpertProduct
from test_rows_abi import fake

ROWS, M, D, EXPERTS = 8, 16, 24, 3


def product(**kw):
    return ExpertProduct(ROWS, M, D, EXPERTS, dtype=torch.float32, device="cpu", **kw)


def call(op, behind_gate):
    op.input_grad(fake(ROWS, M), fake(EXPERTS, M, D), fake(EXPERTS + 1, dtype=torch.int64), saved=fake(ROWS, 2 * D) if behind_gate else None)


@pytest.mark.parametrize("behind_gate", [False, True], ids=["plain", "behind gate"])
@pytest.mark.parametrize("other", [False, True], ids=["alone", "beside the other width"])
@pytest.mark.parametrize("shape", [(ROWS, D + 1), (ROWS, 2 * D - 1), (ROWS + 1, D), (ROWS - 1, 2 * D), (ROWS * D,), (1, ROWS, D), (0, D)])
def test_a_gradient_of_another_shape(shape, other, behind_gate):
    op = product()
    if other:
        op._out("dX", torch.Size((ROWS, 2 * D if behind_gate else D)), torch.float32)
    op.dX = mine = torch.empty(shape)
    with pytest.raises(TypeError, match="dX must be of shape"):
        call(op, behind_gate)
    assert op.dX is mine


@pytest.mark.parametrize("behind_gate", [False, True], ids=["plain", "behind gate"])
def test_a_gradient_of_another_type(behind_gate):
    op = product()
    op.dX = torch.empty(ROWS, 2 * D if behind_gate else D, dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="dX must be of shape"):
        call(op, behind_gate)


def test_the_two_widths_have_a_buffer_each():
    op = product()
    narrow, wide = torch.Size((ROWS, D)), torch.Size((ROWS, 2 * D))
    op.dX = mine = torch.empty(narrow)
    a = op._out("dX", wide, torch.float32)
    assert op.dX is a and a.shape == wide and op._out("dX", narrow, torch.float32) is mine and op._out("dX", wide, torch.float32) is a
    op.dX = later = torch.empty(wide)      # (the narrow one is let go, and so is the wide one before this)
    assert op._out("dX", wide, torch.float32) is later
    b = op._out("dX", narrow, torch.float32)
    assert b.shape == narrow and op.dX is b and op._out("dX", wide, torch.float32) is later
