"""The distillation loss without a gradient, for more rows than a grid has workgroups."""
import pytest
import torch

from paper_2605_08793_amd.rows import RowDistill

pytestmark = pytest.mark.gpu


def test_a_workgroup_goes_on_to_further_rows():
    """4.2 million rows that four waves share: the loss's sums of one row must not meet the maxima of the workgroup's next.
    Eight different rows over and over; 1024 of them on their own, which the same teams take, give the bits."""
    n, m, k, few = (1 << 22) + 301, 2052, 3, 1024
    gen = torch.Generator(device="cuda").manual_seed(7)
    kinds = torch.randn(8, m, generator=gen, device="cuda") * torch.tensor([0.1, 0.5, 1.0, 2.0, 4.0, 8.0, 16.0, 32.0], device="cuda")[:, None]
    columns = torch.randint(0, m, (8, k), generator=gen, device="cuda", dtype=torch.int32)
    given = torch.randn(8, k, generator=gen, device="cuda")
    which = torch.arange(n, device="cuda") % 8

    want = RowDistill(few, m, k, dtype=torch.float32, grad=False)
    want.distill(kinds[which[:few]], columns[which[:few]], given[which[:few]])
    S = torch.empty(n, m, device="cuda")
    for r in range(8):
        S[r::8] = kinds[r]
    op = RowDistill(n, m, k, dtype=torch.float32, grad=False)
    op.loss.fill_(5.0)
    op.distill(S, columns[which], given[which])
    assert torch.equal(op.loss, want.loss[:8][which])
    del S
    torch.cuda.empty_cache()
