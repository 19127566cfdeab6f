"""Routing and its gradient against plain 64-bit ones.

Weights: a score is off by 16 U relative (softmax: exponent 2 U d, exponential and quotient 2 U each, sum of m terms; d <= 40
here), a renormalised one by as much again; with a bias, keys that lie within 8 U of each other may swap, so the chosen
keys are compared as numbers; without one, and on scores alone, the order is exact."""
import numpy as np
import pytest
import torch

import rows_reference as ref
from paper_2605_08793_amd import binding as B
from paper_2605_08793_amd.rows import RowRoute
from rows_reference import TYPE_IDS, TYPES, U, close

pytestmark = pytest.mark.gpu


def weights(S, idx, score, renorm, scale):
    s = ref.route_scores(S, score)
    at = idx.clamp(min=0)
    c = torch.where(idx >= 0, s.gather(1, at), 0.0)
    total = c.sum(1, keepdim=True)
    return scale * (torch.where(total > 0, c / total, 0.0) if renorm else c)


def tol_scores(S):
    x = S.detach().cpu().double()
    fin = torch.where(torch.isfinite(x), x, 0.0)
    d = (fin.amax(1) - fin.amin(1))[:, None] + fin.abs().amax(1, keepdim=True)
    return U * (4 * d + S.shape[1] / 16 + 32)  # relative


def route(S, k, bias=None, bias_on=None, **kw):
    op = RowRoute(S.shape[0], S.shape[1], k, bias_on=bias_on, dtype=S.dtype, **kw)
    op.idx.fill_(-7)
    op.weight.fill_(12345.0)
    op.route(S, bias=bias)
    torch.cuda.synchronize()
    return op


def check(S, op, k, bias, bias_on, score, groups, kept, group_by, renorm, scale, what):
    key, gap = ref.route_keys(S, bias, bias_on, score, groups, kept, group_by)
    exact = bias is None
    assert exact or gap > 1e-5, "the inputs leave a choice of groups to the last bit"
    want_idx, want_key = ref.best(key, k)
    idx = op.idx.cpu().long()
    assert torch.equal(idx < 0, want_idx < 0), what
    if exact:
        assert torch.equal(idx, want_idx), what
    got_key = torch.where(idx >= 0, key.gather(1, idx.clamp(min=0)), -np.inf)
    size = torch.where(torch.isfinite(want_key), want_key.abs(), 0.0)
    close(got_key, want_key, 16 * U * (1 + size) + tol_scores(S), what + " keys")
    for i in range(idx.shape[0]):
        some = idx[i][idx[i] >= 0]
        assert some.unique().numel() == some.numel(), what + ": a column twice"
    w = weights(S, idx, score, renorm, scale)
    close(op.weight, w, w.abs() * (2 * tol_scores(S) + U * (k + 8)) + 1e-36, what + " weights")


def inputs(n, m, dtype, seed, bias):
    g = torch.Generator().manual_seed(seed)
    S = torch.randn(n, m, generator=g).to(dtype)
    return S, (torch.randn(m, generator=g) * bias).float() if bias else None


SHAPES = [(1, 1, 1), (3, 2, 2), (5, 8, 2), (100, 16, 4), (7, 17, 5), (1000, 60, 4), (9, 63, 8), (130, 64, 6), (33, 65, 1), (1, 256, 8),
          (500, 256, 8), (20, 257, 16), (40, 511, 10), (9, 1000, 32), (3, 1024, 32),
          (70, 32, 20), (40, 64, 32), (4100, 64, 3), (5000, 128, 8), (4200, 101, 20), (4096, 127, 4), (30, 300, 32), (50, 512, 3)]


@pytest.mark.parametrize("n,m,k", SHAPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
def test_sizes(n, m, k, score, dtype):
    for bias_on, size in ((None, 0.0), ("score", 0.1), ("logit", 0.5)):
        S, bias = inputs(n, m, dtype, n + m, size)
        for renorm in (True, False):
            op = route(S.cuda(), k, None if bias is None else bias.cuda(), bias_on, score=score, renormalise=renorm, scale=1.5)
            check(S, op, k, bias, bias_on, score, 1, 1, "max", renorm, 1.5, f"{n}x{m} {bias_on} {renorm}")


@pytest.mark.parametrize("m,groups,kept,k", [(8, 4, 2, 3), (60, 6, 2, 5), (64, 64, 10, 8), (256, 8, 4, 8), (256, 8, 8, 8), (96, 3, 1, 20), (1024, 32, 5, 32),
                                             (160, 8, 3, 6), (990, 9, 4, 12), (64, 8, 3, 8), (32, 32, 9, 4), (512, 8, 4, 10), (333, 3, 2, 5), (111, 37, 20, 9),
                                             (480, 60, 13, 17)])
@pytest.mark.parametrize("group_by", ["max", "top2"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_groups(m, groups, kept, k, group_by, score):
    for bias_on, size in ((None, 0.0), ("score", 0.1), ("logit", 0.5)):
        for seed in range(20):  # (the first seed whose group values are apart)
            S, bias = inputs(60, m, torch.float32, m + 100 * seed, size)
            if ref.route_keys(S, bias, bias_on, score, groups, kept, group_by)[1] > 1e-5:
                break
        op = route(S.cuda(), k, None if bias is None else bias.cuda(), bias_on, score=score, groups=groups, groups_kept=kept, group_by=group_by)
        check(S, op, k, bias, bias_on, score, groups, kept, group_by, True, 1.0, f"{m} in {groups}, {bias_on}")


@pytest.mark.parametrize("m,groups,kept,k", [(128, 8, 4, 8), (120, 15, 4, 20), (72, 3, 1, 3), (100, 50, 11, 6)])
@pytest.mark.parametrize("group_by", ["max", "top2"])
def test_groups_of_many_rows(m, groups, kept, k, group_by):
    # each row is copied 90 times, so that the group values of 50 rows have to be apart
    for seed in range(20):
        S, bias = inputs(50, m, torch.float32, m + 100 * seed, 0.1)
        if ref.route_keys(S, bias, "score", "sigmoid", groups, kept, group_by)[1] > 1e-5:
            break
    S = S.repeat(90, 1)
    op = route(S.cuda(), k, bias.cuda(), "score", score="sigmoid", groups=groups, groups_kept=kept, group_by=group_by)
    check(S, op, k, bias, "score", "sigmoid", groups, kept, group_by, True, 1.0, f"{m} in {groups}")


def test_ties_go_to_the_lower_index():
    S = torch.zeros(3, 40)
    S[1, 20:] = 1.0
    S[2, ::7] = 2.0
    for m_kw in (dict(), dict(groups=4, groups_kept=2), dict(groups=4, groups_kept=2, group_by="top2")):
        for score in ("softmax", "sigmoid"):
            op = route(S.cuda(), 6, score=score, **m_kw)
            key, _ = ref.route_keys(S, None, None, score, m_kw.get("groups", 1), m_kw.get("groups_kept", 1), m_kw.get("group_by", "max"))
            assert torch.equal(op.idx.cpu().long(), ref.best(key, 6)[0]), (m_kw, score)
    assert route(S.cuda(), 6).idx[0].tolist() == [0, 1, 2, 3, 4, 5]
    bias = torch.zeros(40).cuda()
    assert route(S.cuda(), 6, bias, "score").idx.tolist() == route(S.cuda(), 6).idx.tolist()


def test_saturated_scores_keep_the_order_of_the_logits():
    S = torch.tensor([[30.0, 40.0, 20.0, -50.0, 25.0]])
    assert route(S.cuda(), 4, score="sigmoid").idx.tolist() == [[1, 0, 4, 2]]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
def test_masks(score, dtype):
    n, m, k = 7, 48, 6
    S, bias = inputs(n, m, dtype, 3, 0.2)
    S[0, 5:] = -np.inf                 # fewer than k left
    S[1] = -np.inf                     # none left
    S[2, ::2] = torch.finfo(dtype).min
    S[3, 8:] = -np.inf                 # one group left
    bias[47] = -np.inf                 # a column out of service
    S[4, 47] = 20.0
    for kw in (dict(), dict(groups=6, groups_kept=2, group_by="top2"), dict(groups=6, groups_kept=2, group_by="max")):
        for b, on in ((None, None), (bias, "score"), (bias, "logit")):
            op = route(S.cuda(), k, None if b is None else b.cuda(), on, score=score, **kw)
            check(S, op, k, b, on, score, kw.get("groups", 1), kw.get("groups_kept", 1), kw.get("group_by", "max"), True, 1.0, f"{kw} {on}")
            assert op.idx[1].tolist() == [-1] * k and op.weight[1].tolist() == [0.0] * k


def test_rows_without_a_number():
    S = torch.randn(4, 32)
    S[0, 31] = np.nan
    S[1, 4] = np.inf
    op = route(S.cuda(), 4)
    for i in (0, 1):
        assert op.idx[i].tolist() == [-1] * 4 and op.weight[i].isnan().all()
    assert (op.idx[2:] >= 0).all() and torch.isfinite(op.weight[2:]).all()
    op = route(S.cuda(), 4, score="sigmoid")
    assert op.idx[0].tolist() == [-1] * 4 and op.weight[0].isnan().all()
    assert op.idx[1, 0] == 4 and torch.isfinite(op.weight[1]).all()


def test_scores_that_vanish():
    S = torch.full((2, 20), -200.0)
    op = route(S.cuda(), 3, score="sigmoid")
    assert op.weight.tolist() == [[0.0] * 3] * 2 and op.idx[0].tolist() == [0, 1, 2]
    assert op.grad(S.cuda(), torch.ones(2, 3, device="cuda")).abs().max() == 0


def grad_reference(S, idx, g, score, renorm, scale):
    s = ref.route_scores(S, score)
    n, m = s.shape
    is_ = (idx >= 0) & (idx < m)
    at = idx.clamp(0, m - 1)
    g = torch.where(is_, g.cpu().double() * scale, 0.0)
    c = torch.where(is_, s.gather(1, at), 0.0)
    size = g.abs()
    if renorm:
        Z = c.sum(1, keepdim=True)
        mean = torch.where(Z > 0, (g * c).sum(1, keepdim=True) / Z, 0.0)
        size = torch.where(is_ & (Z > 0), (g.abs() + (g.abs() * c).sum(1, keepdim=True) / Z) / Z, 0.0)
        g = torch.where(is_ & (Z > 0), (g - mean) / Z, 0.0)
    ds = torch.zeros_like(s).scatter_add_(1, at, g)
    ds_size = torch.zeros_like(s).scatter_add_(1, at, size)
    if score == "softmax":
        d, d_size = s * (ds - (g * c).sum(1, keepdim=True)), s * (ds_size + (size * c).sum(1, keepdim=True))
    else:
        d, d_size = ds * s * (1 - s), ds_size * s
    return d, d_size * (4 * tol_scores(S) + U * (8 * idx.shape[1] + 32)) + 1e-36


@pytest.mark.parametrize("n,m,k", SHAPES)
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
def test_gradient(n, m, k, dtype):
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            S, _ = inputs(n, m, dtype, n * m, 0.0)
            op = route(S.cuda(), k, score=score, renormalise=renorm, scale=2.5)
            g = torch.randn(n, k, generator=torch.Generator().manual_seed(n)).cuda()
            want, tol = grad_reference(S, op.idx.cpu().long(), g, score, renorm, 2.5)
            close(op.grad(S.cuda(), g), want, ref.rounded(want, tol, dtype), f"{n}x{m} {score} {renorm}")


def test_gradient_of_given_choices():
    """Choices from elsewhere: missing ones, none at all, out of range, one twice; rows apart in memory."""
    n, m, k = 6, 70, 5
    S, _ = inputs(n, m, torch.float32, 1, 0.0)
    S[4, 30:] = -np.inf
    S[5] = -np.inf
    idx = torch.randint(0, 30, (n, k), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    idx[0, 2:] = -1
    idx[1] = -1
    idx[2, 0], idx[2, 1] = m, 2 ** 30
    idx[3] = 11
    g = torch.randn(n, k, generator=torch.Generator().manual_seed(2)).cuda()
    wide = torch.full((n, m + 9), float("nan"), device="cuda")
    wide[:, 3:3 + m] = S.cuda()
    out = torch.full((n, m + 5), 7.0, device="cuda")
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            B.regot_row_route_grad(wide[:, 3:3 + m], idx.cuda(), g, out[:, 1:1 + m], score=score, renormalise=renorm, scale=0.5)
            want, tol = grad_reference(S, idx.long(), g, score, renorm, 0.5)
            close(out[:, 1:1 + m], want, ref.rounded(want, tol, torch.float32), f"{score} {renorm}")
            assert (out[:, 0] == 7.0).all() and (out[:, 1 + m:] == 7.0).all()


def test_gradient_against_differences():
    n, m, k = 3, 40, 6
    S, _ = inputs(n, m, torch.float32, 4, 0.0)
    g = torch.randn(n, k, generator=torch.Generator().manual_seed(3)).cuda()
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            op = route(S.cuda(), k, score=score, renormalise=renorm, scale=1.5)
            out, idx = op.grad(S.cuda(), g).cpu().double(), op.idx.cpu().long()
            value = lambda x: float((g.cpu().double() * weights(x, idx, score, renorm, 1.5)).sum())  # noqa: E731
            _, tol = grad_reference(S, idx, g, score, renorm, 1.5)
            rng = torch.Generator().manual_seed(5)
            for _ in range(4):
                v = torch.randn(n, m, generator=rng, dtype=torch.float64)
                step = 1e-4
                slope = (value(S.double() + step * v) - value(S.double() - step * v)) / (2 * step)
                assert abs(float((out * v).sum()) - slope) <= float((ref.rounded(out, tol, torch.float32) * v.abs()).sum()) + 1e-5


def test_many_rows_and_none():
    S, bias = inputs(70_001, 32, torch.bfloat16, 6, 0.0)
    op = route(S.cuda(), 4)
    assert torch.equal(op.idx.cpu().long(), ref.best(S.double(), 4)[0])
    op = route(torch.empty(3, 0, device="cuda"), 2)
    assert (op.idx == -1).all() and (op.weight == 0).all()
    route(torch.empty(0, 8, device="cuda"), 2)


def test_rows_apart():
    n, m = 50, 100
    S, bias = inputs(n, m, torch.bfloat16, 2, 0.0)
    for offset, ld in ((0, 101), (1, 100), (3, 107)):
        flat = torch.full((offset + n * ld,), float("nan"), dtype=torch.bfloat16, device="cuda")
        view = flat[offset:].view(n, ld)[:, :m]
        view.copy_(S)
        assert torch.equal(route(view, 7).idx.cpu().long(), ref.best(S.double(), 7)[0])
