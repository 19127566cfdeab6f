"""Products and gradients of 32-bit numbers over the whole range of 32 bits: numbers near the smallest, below it, and near the largest, alone and beside ordinary ones.

A sum of c products is off by at most (c + 16) 2 U times the sum of their sizes, as everywhere: c + 16 times a rounding or a cut of what has been added up so far.  Below the smallest
normal number such a rounding is one to a multiple of 2^-149 instead, so c + 16 of these are added.  Where the sizes add up to more than the largest number of 32 bits, an
addition on the way may overflow whatever the whole sum is, in any order that has the numbers of one sign first: such a result may be anything."""
import pytest
import torch

from paper_2605_08793_amd import binding as B
from rows_reference import U

pytestmark = pytest.mark.gpu
STEP = 2.0 ** -149
# sizes of the two sides: products that are ordinary numbers, small ones, below the smallest normal number; numbers that are themselves below it; large ones
SCALES = [(1e-36, 1e10), (1e-37, 1e36), (1e-41, 1e20), (1e-44, 1e30), (1.0, 1e-36), (1e10, 1e-38), (1e-20, 1e-15), (1e-25, 1e-17), (1e32, 1.0), (1e36, 1e-36), (1e30, 1e5), (1e-30, 1e37)]
IDS = [f"{a:g} by {b:g}" for a, b in SCALES]


def bound(size, count):
    tol = (size * 2 * U + STEP) * (count + 16)
    return torch.where(size < torch.finfo(torch.float32).max, tol, float("inf"))


def close(got, want, tol, what):
    sure = tol < float("inf")
    off, tol = (got.cpu().double() - want).abs()[sure], tol[sure]
    assert bool((off <= 1.01 * tol).all()), f"{what}: {float((off / tol).max()):.3g} times the bound"


def normal(gen, *shape):
    """Of sizes between 1/2 and 4, so that nothing leaves the range by itself."""
    return (torch.rand(*shape, generator=gen) * 3.5 + 0.5) * (torch.randint(0, 2, shape, generator=gen) * 2 - 1)


@pytest.mark.parametrize("rows,d,m", [(9, 64, 40), (200, 64, 40), (200, 33, 17), (150, 512, 136)])
@pytest.mark.parametrize("turned", [False, True], ids=["outputs", "inputs"])
@pytest.mark.parametrize("scale,by", SCALES, ids=IDS)
def test_products_and_gradients(scale, by, turned, rows, d, m):
    """Every third row is an ordinary one (its results are those of an ordinary row by the scaled weights)."""
    gen = torch.Generator().manual_seed(rows + d)
    X, dY = normal(gen, rows, d), normal(gen, rows, m)
    for t in (X, dY):
        t[torch.arange(rows) % 3 != 0] *= scale
    W = normal(gen, 1, m, d) * by
    start, V = torch.tensor([0, rows], device="cuda"), W.transpose(1, 2).contiguous().cuda().transpose(1, 2) if turned else W.cuda()
    x, g, w = X.double(), dY.double(), W[0].double()

    Y = torch.empty(rows, m, device="cuda")
    B.regot_expert_product(X.cuda(), V, start, Y)
    close(Y, x @ w.t(), bound(x.abs() @ w.abs().t(), d), "Y")
    dX = torch.empty(rows, d, device="cuda")
    B.regot_expert_product(dY.cuda(), V.transpose(1, 2), start, dX)
    close(dX, g @ w, bound(g.abs() @ w.abs(), m), "dX")

    X, dY = normal(gen, rows, d) * scale, normal(gen, rows, m) * by
    dW = torch.empty(1, m, d, device="cuda")
    ws = torch.empty(B.regot_expert_weight_grad_workspace_bytes(rows, m, d, 1), dtype=torch.uint8, device="cuda")
    B.regot_expert_weight_grad(dY.cuda(), X.cuda(), start, dW, workspace=ws)
    close(dW[0], dY.double().t() @ X.double(), bound(dY.double().abs().t() @ X.double().abs(), rows), "dW")


@pytest.mark.parametrize("d", [64, 33])
@pytest.mark.parametrize("scale,by", [(1e-36, 1e35), (1e-41, 1e38), (1e34, 1e-34)])
def test_gate(scale, by, d):
    """What is kept before the gate, and the gradient to it: gates of 0, so that s(g) = 1/2 whatever the sums are."""
    rows, m = 100, 40
    gen = torch.Generator().manual_seed(d)
    X, W = normal(gen, rows, d) * scale, normal(gen, 1, 2 * m, d) * by
    start = torch.tensor([0, rows], device="cuda")
    Y, saved = torch.empty(rows, m, device="cuda"), torch.empty(rows, 2 * m, device="cuda")
    B.regot_expert_product(X.cuda(), W.cuda(), start, Y, act="gate", saved=saved)
    x, w = X.double(), W[0].double()
    close(saved, x @ w.t(), bound(x.abs() @ w.abs().t(), d), "saved")
    at = torch.zeros(rows, 4 * m)
    at[:, 2 * m:] = normal(gen, rows, 2 * m)
    dX = torch.empty(rows, 4 * m, device="cuda")
    B.regot_expert_product(X.cuda(), W.cuda(), start, dX, act="gate_grad", saved=at.cuda())
    D, t, u = x @ w.t(), bound(x.abs() @ w.abs().t(), d), at[:, 2 * m:].double()
    close(dX[:, :2 * m], D * u / 2, (t * u.abs() + 2 * U * (D * u).abs()) / 2 + STEP, "dg")
    assert bool((dX[:, 2 * m:].cpu()[t < float("inf")] == 0).all())       # (0 times an infinity is none)


def test_few_finite_numbers_that_overflow_between():
    """Sums that are within 32 bits though the first products alone are not are what 32-bit arithmetic makes of them, and the rows beside them as they are alone."""
    gen = torch.Generator().manual_seed(0)
    X, W = normal(gen, 70, 64), normal(gen, 1, 40, 64)
    start = torch.tensor([0, 70], device="cuda")
    alone, beside = torch.empty(70, 40, device="cuda"), torch.empty(70, 40, device="cuda")
    B.regot_expert_product(X.cuda(), W.cuda(), start, alone)
    Z = X.clone()
    Z[11] *= 1e38
    B.regot_expert_product(Z.cuda(), W.cuda(), start, beside)
    assert torch.equal(beside[:11], alone[:11]) and torch.equal(beside[12:], alone[12:])
