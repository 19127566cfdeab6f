"""Rows that hold a NaN or +inf have no gradient: NaN at every column, at the choices that routing gives them (none) and at given ones."""
import numpy as np
import pytest
import torch

from paper_2605_08793_amd import binding as B
from paper_2605_08793_amd.rows import RowRoute
from rows_reference import TYPE_IDS, TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("m", [5, 32, 64, 100, 256, 500, 1000])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
def test_the_gradient_is_nan_too(score, renormalise, m, dtype):
    n, k = 71, 3
    S = torch.randn(n, m, generator=torch.Generator().manual_seed(m)).to(dtype)
    nan, inf, empty = [0, 13, 70], [4, 30], [8, 69]
    for i, j in zip(nan, (0, m // 2, m - 1)):
        S[i, j] = np.nan
    S[inf, m // 3] = np.inf
    S[empty] = -np.inf
    S[13, 0] = -np.inf
    without = nan + (inf if score == "softmax" else [])
    g = torch.randn(n, k, generator=torch.Generator().manual_seed(1)).cuda()
    op = RowRoute(n, m, k, score=score, renormalise=renormalise, dtype=dtype)
    op.route(S.cuda())
    assert op.weight[without].isnan().all() and (op.idx[without] == -1).all()
    given = torch.randint(0, m, (n, k), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    given[5] = -1
    given[13] = -1
    given[6, 1:] = -1
    out = torch.full((n, m), 7.0, dtype=dtype, device="cuda")
    B.regot_row_route_grad(S.cuda(), given.cuda(), g, out, score=score, renormalise=renormalise)
    for d in (op.grad(S.cuda(), g), out):
        assert d[without].isnan().all()
        others = [i for i in range(n) if i not in without]
        assert torch.isfinite(d[others]).all()
        assert (d[empty] == 0).all()
    assert (out[5] == 0).all()
    assert (out[6] != 0).any() or renormalise      # (one renormalised choice has the weight 1 whatever the scores are)


def test_a_nan_in_the_bias():
    S = torch.randn(4, 32).cuda()
    bias = torch.zeros(32)
    bias[7] = np.nan
    op = RowRoute(4, 32, 3, bias_on="logit")
    op.route(S, bias=bias.cuda())
    assert (op.idx == -1).all() and op.weight.isnan().all()
    assert (op.grad(S, torch.ones(4, 3, device="cuda")) == 0).all()
