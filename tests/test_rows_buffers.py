"""The buffers of the row objects: made without a launch, and not to be replaced, since a call writes to those it was made with."""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2605_08793_amd.rows import RowDistill, RowLogprob, RowRoute

OUTPUTS = [(lambda: RowLogprob(4, 9, k=3, targets=2, device="cpu"), ["logprob_out", "entropy", "stats", "top_idx", "top_logprob", "workspace"]),
           (lambda: RowDistill(4, 9, 3, device="cpu"), ["loss", "grad", "workspace"]),
           (lambda: RowRoute(4, 9, 3, device="cpu"), ["idx", "weight"])]


class Seen(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.names = set()

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        self.names.add(func.overloadpacket.__name__)
        return func(*args, **(kwargs or {}))


@pytest.mark.parametrize("make,names", OUTPUTS, ids=["logprob", "distill", "route"])
def test_outputs_are_not_replaced(make, names):
    op = make()
    for name in names:
        with pytest.raises(AttributeError):
            setattr(op, name, torch.empty(4, 9))
        assert isinstance(getattr(op, name), torch.Tensor)


@pytest.mark.parametrize("make,names", OUTPUTS, ids=["logprob", "distill", "route"])
def test_nothing_is_filled(make, names):
    with Seen() as seen:
        make()
    assert seen.names == {"empty"}


def test_shapes_and_what_is_left_out():
    op = RowLogprob(4, 9, targets=0, device="cpu")
    assert op.logprob_out is None and op.top_idx is None and op.top_logprob is None and op.dS is None
    assert op.entropy.shape == (4,) and op.stats.shape == (4, 2)
    assert RowDistill(4, 9, 3, grad=False, device="cpu").grad is None
    op.dS = torch.empty(4, 9)      # (what `grad` writes to, if it is of the scores' shape, type and device)
    assert op.dS.shape == (4, 9)
