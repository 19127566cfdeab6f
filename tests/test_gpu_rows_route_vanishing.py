"""Renormalised weights, and their gradient, where the chosen scores are near the smallest 32-bit numbers: a quotient of them is
an ordinary number, scale / sum and g / sum are not.

Bound, U = 2^-24: a score is off by U (|x| + 6) relative for sigmoid (exponent's argument U |x|, exponential and reciprocal 2 U each, sum U) and by
U (2 d + m / 16 + 32) for softmax, d the distance from the maximum; a quotient of two of them by twice that and 4 U, sums of k terms by k U."""
import pytest
import torch

from paper_2605_08793_amd.rows import RowRoute
from rows_reference import U, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [1.0, 16.0, 1e6])
@pytest.mark.parametrize("m,k", [(20, 1), (30, 3), (64, 8), (200, 8), (600, 20)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_the_smallest_scores(score, m, k, scale):
    far = torch.arange(78.0, 87.0, 0.25)                       # (e^-87 is above the smallest normal number, 2^-126)
    n = len(far)
    S = torch.full((n, m), -200.0)
    chosen = 5 + torch.arange(k)
    S[:, chosen] = -far[:, None] - 0.3 * torch.rand(n, k, generator=torch.Generator().manual_seed(k))
    bias = torch.zeros(m)
    if score == "softmax":
        S[:, 2] = 0.0                                          # (which has all of the distribution, and is not chosen)
        bias[chosen] = 300.0
    op = RowRoute(n, m, k, score=score, bias_on="logit", scale=scale)
    op.route(S.cuda(), bias=bias.cuda())
    g = torch.randn(n, k, generator=torch.Generator().manual_seed(m), dtype=torch.float64).float()
    idx = op.idx.cpu().long()
    assert torch.equal(idx.sort(1).values, chosen.repeat(n, 1))
    x = S.double()
    s = torch.softmax(x, 1) if score == "softmax" else torch.sigmoid(x)
    c = s.gather(1, idx)
    w = c / c.sum(1, keepdim=True)
    tol = U * (2 * (2 * 88 + m / 16 + 32) + k + 8)
    close(op.weight, scale * w, scale * w * tol, "weights")
    G = scale * g.double()
    mean = (G * w).sum(1, keepdim=True)
    part = (G - mean) * w * ((1 - c) if score == "sigmoid" else 1.0)
    size = (G.abs() + (G.abs() * w).sum(1, keepdim=True)) * w
    d = torch.zeros(n, m, dtype=torch.float64).scatter_(1, idx, part)
    bound = torch.zeros(n, m, dtype=torch.float64).scatter_(1, idx, size * (2 * tol + 8 * U))
    if score == "softmax":
        d -= s * part.sum(1, keepdim=True)
        bound += s * (size.sum(1, keepdim=True) * (2 * tol + 8 * U))
    close(op.grad(S.cuda(), g.cuda()), d, bound + 2.0 ** -126, "gradient")
