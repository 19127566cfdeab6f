"""The order of choices by expert, and the weighted sum of the experts' rows with its gradients, against plain 64-bit arithmetic."""
import numpy as np
import pytest
import torch

import experts_reference as ref
from paper_2605_08793_amd.experts import ExpertCombine, ExpertOrder
from rows_reference import TYPES, TYPE_IDS

pytestmark = pytest.mark.gpu


def check_order(idx, experts):
    n, k = idx.shape
    op = ExpertOrder(n, k, experts)
    for t in (op.start, op.order, op.place):
        t.fill_(77)
    op.sort(idx.cuda())
    for got, want, what in zip((op.start, op.order, op.place), ref.order(idx, experts), ("start", "order", "place")):
        np.testing.assert_array_equal(got.cpu().numpy(), want.numpy(), err_msg=what)


SIZES = [(0, 3, 5), (1, 1, 1), (1, 8, 256), (1, 1, 1024), (63, 1, 2), (64, 2, 3), (65, 3, 1000), (1000, 4, 60), (513, 7, 31), (4096, 4, 16), (4097, 4, 64),
         (16384, 1, 1024), (16385, 1, 1024), (30000, 8, 256), (70001, 32, 9), (600000, 8, 128), (5, 2, 0)]


@pytest.mark.parametrize("n,k,experts", SIZES)
def test_order(n, k, experts):
    gen = torch.Generator().manual_seed(n + 10 * k + 100 * experts)
    idx = ref.choices(n, k, experts, gen) if experts else torch.full((n, k), -1, dtype=torch.int32)
    check_order(idx, experts)


@pytest.mark.parametrize("n", [50, 5000, 40000])
@pytest.mark.parametrize("what", ["one expert", "none", "alternating", "twice", "outside"])
def test_order_of_special_choices(n, what):
    idx = torch.zeros(n, 2, dtype=torch.int32)
    if what == "one expert":
        idx += 3
    elif what == "none":
        idx -= 1
    elif what == "alternating":
        idx += torch.arange(n, dtype=torch.int32)[:, None] % 5
    elif what == "outside":
        idx[::3, 0], idx[1::3, 1], idx[2::3, 1] = 2 ** 31 - 1, -2 ** 31, 5
    check_order(idx, 5)


COMBINE = [(1, 1, 1, 0.0), (1, 8, 2048, 0.0), (3, 2, 7, 0.3), (64, 4, 513, 0.2), (100, 5, 64, 0.5), (33, 32, 130, 0.1), (257, 3, 1000, 1.0), (2000, 6, 96, 0.1)]


def rows_of(n, k, m, dtype, seed, dropped, stride=0):
    gen = torch.Generator().manual_seed(seed)
    idx = ref.choices(n, k, 6, gen, dropped)
    _, _, place = ref.order(idx, 6)
    rows = n * k + 3

    def matrix(count):
        wide = torch.full((count, m + stride), float("nan"), dtype=dtype)
        wide[:, :m] = torch.randn(count, m, generator=gen).to(dtype)
        return wide.cuda()[:, :m]

    weight = torch.rand(n, k, generator=gen) * 2 - 0.5
    return place, matrix(rows), matrix(n), weight, rows


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("stride", [0, 5])
@pytest.mark.parametrize("n,k,m,dropped", COMBINE)
def test_combine_and_gradients(n, k, m, dropped, stride, dtype):
    place, Y, g_out, weight, rows = rows_of(n, k, m, dtype, n + m, dropped, stride)
    op = ExpertCombine(n, k, m, rows=rows, dtype=dtype)
    for w in (weight, None):
        on = None if w is None else w.cuda()
        wide = None if w is None else w.double()
        op.combine(Y, place.cuda(), on)
        want, tol = ref.combine(Y.cpu().double(), place, wide)
        ref.close(op.out, want, ref.rounded(want, tol, dtype), "out")
        op.dY = torch.full((rows, m), 5.0, dtype=dtype, device="cuda")
        op.grad(g_out, Y, place.cuda(), on)
        dY, t_dY, gw, t_gw = ref.combine_grad(g_out.cpu().double(), Y.cpu().double(), place, wide, rows)
        nobody = dY.isnan()
        assert bool((op.dY.cpu()[nobody] == 5.0).all())
        ref.close(op.dY.cpu()[~nobody], dY[~nobody], ref.rounded(dY, t_dY, dtype)[~nobody], "dY")
        ref.close(op.g_weight, gw, t_gw, "g_weight")
        before = op.g_weight.clone()
        op.dY.fill_(5.0)
        op.grad(g_out, None, place.cuda(), on)
        ref.close(op.dY.cpu()[~nobody], dY[~nobody], ref.rounded(dY, t_dY, dtype)[~nobody], "dY without Y")
        assert torch.equal(before, op.g_weight)


def test_combine_gradient_against_differences():
    """32-bit rows; out is linear in Y and in the weights, so a difference has no error but the roundings of the two sums."""
    n, k, m = 7, 3, 20
    place, Y, g_out, weight, rows = rows_of(n, k, m, torch.float32, 3, 0.2)
    op = ExpertCombine(n, k, m, rows=rows, dtype=torch.float32)
    place, weight = place.cuda(), weight.cuda()
    op.grad(g_out, Y, place, weight)
    dY, gw = op.dY.clone(), op.g_weight.clone()

    def total(Y, weight):
        op.combine(Y, place, weight)
        return float((op.out.double() * g_out.double()).sum())

    size = float((g_out.double().abs().sum())) * 20 * 2.0 ** -23
    gen = torch.Generator(device="cuda").manual_seed(1)
    step_Y, step_w = torch.randn(rows, m, generator=gen, device="cuda"), torch.randn(n, k, generator=gen, device="cuda")
    live = torch.zeros(rows, dtype=torch.bool, device="cuda")
    live[place[place >= 0].long()] = True
    want = float((dY[live].double() * step_Y[live].double()).sum())
    assert abs((total(Y + step_Y, weight) - total(Y - step_Y, weight)) / 2 - want) < 10 * size
    want = float((gw.double() * step_w.double()).sum())
    assert abs((total(Y, weight + step_w) - total(Y, weight - step_w)) / 2 - want) < 10 * size


def test_infinities_and_missing_rows():
    """A row that nobody has adds nothing whatever its weight is; an infinity reaches the tokens that have its row."""
    op = ExpertCombine(3, 2, 4, rows=4, dtype=torch.float32)
    Y = torch.ones(4, 4, device="cuda")
    Y[1, 2], Y[3] = float("inf"), float("nan")
    place = torch.tensor([[0, -1], [1, 2], [4, -7]], dtype=torch.int32, device="cuda")
    weight = torch.tensor([[2.0, float("nan")], [0.5, 1.0], [float("inf"), float("inf")]], device="cuda")
    op.combine(Y, place, weight)
    assert torch.equal(op.out.cpu(), torch.tensor([[2.0] * 4, [1.5, 1.5, float("inf"), 1.5], [0.0] * 4]))
    op.grad(torch.ones(3, 4, device="cuda"), Y, place, weight)
    assert torch.equal(op.g_weight.cpu(), torch.tensor([[4.0, 0.0], [float("inf"), 4.0], [0.0, 0.0]]))


def test_nothing_to_do():
    for n, m in ((0, 8), (4, 0)):
        op = ExpertCombine(n, 2, m, dtype=torch.float32)
        place = torch.zeros(n, 2, dtype=torch.int32, device="cuda")
        Y = torch.zeros(n * 2, m, device="cuda")
        op.combine(Y, place, None)
        op.g_weight.fill_(3.0)
        op.grad(torch.zeros(n, m, device="cuda"), Y, place, None)
        assert bool((op.g_weight == 0).all())
