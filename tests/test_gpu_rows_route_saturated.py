"""The routing gradient of scores near 1 and near 0: sigmoid's s (1 - s) far from the middle.

Bound: with U = 2^-24, s and 1 - s are each off by U (|x| + 6) relative (the exponent's argument U |x|, the exponential and the
reciprocal 2 U each, the sum U), the product with scale and g 4 U more."""
import pytest
import torch

import rows_reference as ref
from paper_2605_08793_amd import binding as B
from rows_reference import TYPE_IDS, TYPES, U, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("m,k", [(25, 3), (60, 8), (256, 8), (300, 32)])
def test_sigmoid_far_from_the_middle(dtype, m, k):
    logits = [0.0, 4.0, 8.0, 10.0, 12.0, 14.0, 16.0, 17.0, 18.0, 20.0, 25.0, 40.0, 60.0, 80.0]
    logits = torch.tensor(logits + [-x for x in logits])
    n = len(logits)
    S = torch.randn(n, m, generator=torch.Generator().manual_seed(m))
    S[:, 7:7 + k] = logits[:, None] + torch.arange(k) / 8
    S = S.to(dtype)
    idx = (7 + torch.arange(k, dtype=torch.int32)).repeat(n, 1)
    scale = 3.0e4 if dtype == torch.float16 else 2.5
    g = torch.randn(n, k, generator=torch.Generator().manual_seed(k))
    out = torch.full((n, m), 7.0, dtype=dtype, device="cuda")
    B.regot_row_route_grad(S.cuda(), idx.cuda(), g.cuda(), out, score="sigmoid", renormalise=False, scale=scale)
    x = S.double()
    d = torch.zeros(n, m, dtype=torch.float64)
    d.scatter_(1, idx.long(), scale * g.double())
    d *= torch.sigmoid(x) * torch.sigmoid(-x)
    close(out, d, ref.rounded(d, d.abs() * U * (2 * x.abs() + 16), dtype), "gradient")
