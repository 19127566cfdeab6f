"""Runs of large finite negative scores as a mask: a lane, a wave or a part of a row may see nothing else until its sums are
joined.  Bounds in rows_reference."""
import pytest
import torch

import rows_reference as ref
from rows_reference import TYPE_IDS, TYPES, close
from test_gpu_rows_logprob import call, check, gradient, scores, targets_for

pytestmark = pytest.mark.gpu


def closed(kind, S, value):
    m = S.shape[1]
    if kind == "first half":
        S[:, :m // 2] = value
    elif kind == "last columns":
        S[:, m - max(1, min(100, m // 2)):] = value
    elif kind == "all but few":
        kept = torch.tensor(sorted({m // 3, m // 2, m - 1}))
        few = S[:, kept].clone()
        S[:] = value
        S[:, kept] = few
    elif kind == "one column":
        S[:, min(3, m - 1)] = value
    elif kind == "steps":  # each stretch above the one before it
        for i in range(4):
            S[:, i * m // 5:(i + 1) * m // 5] = value / 2 ** (4 * i)
    return S


@pytest.mark.parametrize("kind", ["first half", "last columns", "all but few", "one column", "steps"])
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("m", [2, 64, 100, 128, 300, 1000, 3000, 5003, 20011, 131072])
def test_runs_of_lowest_scores(kind, dtype, m):
    n = 3
    target = targets_for(n, m, 2, 3)
    g, h = torch.full((n, 2), 0.5).cuda(), torch.full((n,), -0.3).cuda()
    least = torch.finfo(dtype).min
    for value in (least, least / 4, least / 32):
        S = closed(kind, scores(n, m, dtype, m), value)
        for eta in (0.5, 1.0, 2.0):
            what = f"{kind} {value:.3g} eta {eta}"
            for k in (0, 5):
                check(call(S.cuda(), target, eta, k), S, target, eta, k, None, what)
            want, tol = ref.logprob_grad(ref.Rows(S, None, eta), target, g, h)
            close(gradient(S, target, eta, None, g, h), want, ref.rounded(want, tol, dtype), what + " gradient")
