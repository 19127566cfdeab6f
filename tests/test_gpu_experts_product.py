"""Products grouped by expert and their gradients against plain 64-bit arithmetic."""
import numpy as np
import pytest
import torch

import experts_reference as ref
from paper_2605_08793_amd import binding as B
from paper_2605_08793_amd.experts import ExpertProduct
from rows_reference import TYPES, TYPE_IDS

pytestmark = pytest.mark.gpu
NAN = float("nan")


def matrix(gen, rows, cols, dtype, gap=0, scale=1.0):
    """rows x cols, with `gap` columns of NaN behind each row that no call may look at."""
    wide = torch.full((rows, cols + gap), NAN, dtype=dtype)
    wide[:, :cols] = (torch.randn(rows, cols, generator=gen) * scale).to(dtype)
    return wide.cuda()[:, :cols]


def weights(gen, experts, outputs, inputs, dtype, gap=0, turned=False):
    """(experts, outputs, inputs), the inputs' or (turned) the outputs' numbers neighbours, NaN in the gaps."""
    a, b = (inputs, outputs) if turned else (outputs, inputs)
    wide = torch.full((experts, a + (1 if gap else 0), b + gap), NAN, dtype=dtype)
    wide[:, :a, :b] = (torch.randn(experts, a, b, generator=gen) * max(inputs, 1) ** -0.5).to(dtype)
    W = wide.cuda()[:, :a, :b]
    return W.transpose(1, 2) if turned else W


class Case:
    def __init__(self, n, k, experts, d, m, dtype, gap=0, turned=False, gated=False, seed=0, dropped=0.1):
        self.gen = gen = torch.Generator().manual_seed(seed + n + 3 * d + 7 * m)
        self.n, self.k, self.experts, self.d, self.m, self.dtype, self.gap, self.gated = n, k, experts, d, m, dtype, gap, gated
        self.rows = n * k
        self.start, self.order, self.place = ref.order(ref.choices(n, k, experts, gen, dropped), experts)
        self.X = matrix(gen, n, d, dtype, gap)
        self.wide = 2 * m if gated else m
        self.W = weights(gen, experts, self.wide, d, dtype, gap, turned)
        self.live = int(self.start[-1])

    def op(self, **kw):
        op = ExpertProduct(self.rows, self.m, self.d, self.experts, gated=self.gated, keep=self.gated, dtype=self.dtype, **kw)
        for t in (op.Y, op.saved):
            if t is not None:
                t.fill_(7.0)
        return op

    def on(self):
        return self.start.cuda(), self.order.cuda(), self.k

    def wide_rows(self):
        return ref.source(self.X.cpu().double(), self.order, self.k)


def same_beyond(t, live, value=7.0):
    assert bool((t[live:] == value).all()), "rows of no expert were written"


SIZES = [(1, 1, 1, 1, 1), (1, 8, 16, 64, 64), (3, 2, 5, 7, 9), (5, 1, 4, 64, 130), (40, 2, 3, 72, 136), (130, 1, 1, 200, 264), (300, 3, 7, 129, 257),
         (257, 2, 40, 96, 40), (600, 2, 3, 320, 272), (64, 4, 60, 1400, 48), (1000, 1, 2, 64, 8), (17, 3, 4, 2048, 16), (2, 2, 300, 40, 24)]


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
@pytest.mark.parametrize("turned", [False, True], ids=["outputs", "inputs"])
@pytest.mark.parametrize("n,k,experts,d,m", SIZES)
def test_product(n, k, experts, d, m, turned, gated, dtype):
    c = Case(n, k, experts, d, m, dtype, turned=turned, gated=gated)
    op = c.op()
    op.product(c.X, c.W, *c.on())
    z, tol = ref.sums(c.wide_rows(), c.W.cpu().double(), c.start)
    h, t = ref.gate(z, tol) if gated else (z, tol)
    ref.close(op.Y[:c.live], h[:c.live], ref.rounded(h, t, dtype)[:c.live], "Y")
    same_beyond(op.Y, c.live)
    if gated:
        ref.close(op.saved[:c.live], z[:c.live], ref.rounded(z, tol, dtype)[:c.live], "saved")
        same_beyond(op.saved, c.live)


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("gap", [0, 3, 8])
@pytest.mark.parametrize("behind_gate", [False, True], ids=["plain", "behind gate"])
@pytest.mark.parametrize("turned", [False, True], ids=["outputs", "inputs"])
@pytest.mark.parametrize("n,k,experts,d,m", SIZES)
def test_gradients(n, k, experts, d, m, turned, behind_gate, gap, dtype):
    c = Case(n, k, experts, d, m, dtype, gap=gap, turned=turned)
    start, order, k = c.on()
    dY = matrix(c.gen, c.rows, m, dtype, gap)
    op = c.op()
    D, tol = ref.sums(dY.cpu().double(), c.W.cpu().double().transpose(1, 2), c.start)
    if behind_gate:
        saved = matrix(c.gen, c.rows, 2 * d, dtype, gap, scale=3.0)
        op.dX = torch.full((c.rows, 2 * d), 7.0, dtype=dtype, device="cuda")
        op.input_grad(dY, c.W, start, saved=saved)
        D, tol = ref.gate_grad(D, tol, saved.cpu().double())
    else:
        op.dX = torch.full((c.rows, d), 7.0, dtype=dtype, device="cuda")
        op.input_grad(dY, c.W, start)
    ref.close(op.dX[:c.live], D[:c.live], ref.rounded(D, tol, dtype)[:c.live], "dX")
    same_beyond(op.dX, c.live)

    for gather in (True, False):
        X = c.X if gather else matrix(c.gen, c.rows, d, dtype, gap)
        rows = c.wide_rows() if gather else X.cpu().double()
        want, tol = ref.weight_grad(dY.cpu().double(), rows, c.start)
        for out in {dtype, torch.float32}:
            op = c.op(grad_dtype=out)
            wide = torch.full((experts, m + 1, d + gap), 7.0, dtype=out, device="cuda")
            op.dW = wide[:, :m, :d]
            op.weight_grad(dY, X, start, order if gather else None, k if gather else 1)
            ref.close(op.dW, want, ref.rounded(want, tol, out), f"dW {out} {gather}")
            assert bool((wide[:, m:] == 7.0).all()) and bool((wide[:, :, d:] == 7.0).all())


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("experts,rows,m,d", [(1, 5000, 128, 200), (2, 3000, 64, 64), (3, 8000, 260, 130)])
def test_long_sums_in_parts(experts, rows, m, d, dtype):
    c = Case(rows, 1, experts, d, m, dtype, dropped=0.0)
    assert B.regot_expert_weight_grad_workspace_bytes(rows, m, d, experts) > 256
    dY = matrix(c.gen, rows, m, dtype)
    want, tol = ref.weight_grad(dY.cpu().double(), c.wide_rows(), c.start)
    for out in {dtype, torch.float32}:
        op = c.op(grad_dtype=out)
        got = [op.weight_grad(dY, c.X, *c.on()).clone() for _ in range(2)]
        ref.close(got[0], want, ref.rounded(want, tol, out), "dW")
        assert torch.equal(*got)


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("d,m", [(64, 64), (72, 40), (33, 17)])
def test_non_finite_numbers_stay_where_they_belong(d, m, dtype):
    """A NaN or an infinity reaches its own row (products) or its own expert (weight gradients), and nothing else."""
    n, experts = 90, 3
    start = torch.tensor([0, 30, 61, 90])
    gen = torch.Generator().manual_seed(d)
    X, dY, W = matrix(gen, n, d, dtype), matrix(gen, n, m, dtype), weights(gen, experts, m, d, dtype)
    clean = ExpertProduct(n, m, d, experts, dtype=dtype)
    clean.product(X, W, start.cuda())
    clean.input_grad(dY, W, start.cuda())
    clean.weight_grad(dY, X, start.cuda())
    X[35, 3], X[60, 0], dY[40, 1] = NAN, float("inf"), -float("inf")
    op = ExpertProduct(n, m, d, experts, dtype=dtype)
    op.product(X, W, start.cuda())
    op.input_grad(dY, W, start.cuda())
    op.weight_grad(dY, X, start.cuda())
    assert bool(op.Y[35].isnan().all()) and not bool(op.Y[60].isfinite().any()) and not bool(op.dX[40].isfinite().any())
    other = torch.ones(n, dtype=torch.bool, device="cuda")
    other[[35, 60]] = False
    assert torch.equal(op.Y[other], clean.Y[other])
    other[:] = True
    other[40] = False
    assert torch.equal(op.dX[other], clean.dX[other])
    assert torch.equal(op.dW[[0, 2]], clean.dW[[0, 2]])
    assert bool(op.dW[1, :, 3].isnan().all()) and not bool(op.dW[1, 1].isfinite().any())
    assert torch.equal(op.dW[1, 2:, 4:], clean.dW[1, 2:, 4:])


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
def test_saturated_gates(dtype):
    """Gates far from 0: silu(g) is g, or 0, and nothing overflows on the way."""
    op = ExpertProduct(2, 8, 8, 1, gated=True, keep=True, dtype=dtype)
    X = torch.zeros(2, 8, dtype=dtype, device="cuda")
    X[0, 0], X[1, 0] = 200.0, -200.0
    W = torch.zeros(1, 16, 8, dtype=dtype, device="cuda")
    W[:, :, 0] = 1.0
    W[:, 8:, 0] = 0.25
    start = torch.tensor([0, 2], device="cuda")
    op.product(X, W, start)
    assert bool((op.Y[0] == 200.0 * 50.0).all()) and bool((op.Y[1] == 0.0).all())
    down = ExpertProduct(2, 8, 8, 1, dtype=dtype)
    eye = torch.eye(8, dtype=dtype, device="cuda")[None]
    dX = down.input_grad(torch.ones(2, 8, dtype=dtype, device="cuda"), eye, start, saved=op.saved)
    assert bool((dX[0, :8] == 50.0).all()) and bool((dX[0, 8:] == 200.0).all()) and bool((dX[1] == 0.0).all())


def test_empty_sums_and_experts():
    start = torch.tensor([0, 0, 5, 5], device="cuda")
    op = ExpertProduct(6, 4, 0, 3, dtype=torch.float32)
    op.Y.fill_(7.0)
    op.product(torch.empty(6, 0, device="cuda"), torch.empty(3, 4, 0, device="cuda"), start)
    assert bool((op.Y[:5] == 0).all()) and bool((op.Y[5] == 7.0).all())
    op = ExpertProduct(6, 4, 8, 3, dtype=torch.float32)
    op.weight_grad(torch.ones(6, 4, device="cuda"), torch.ones(6, 8, device="cuda"), start)
    assert bool((op.dW[[0, 2]] == 0).all()) and bool((op.dW[1] == 5.0).all())
    none = ExpertProduct(0, 4, 8, 3, dtype=torch.float32)
    zero = torch.zeros(4, dtype=torch.int64, device="cuda")
    none.product(torch.empty(0, 8, device="cuda"), torch.ones(3, 4, 8, device="cuda"), zero)
    none.weight_grad(torch.empty(0, 4, device="cuda"), torch.empty(0, 8, device="cuda"), zero)
    assert bool((none.dW == 0).all())


def test_starts_outside_the_rows_are_not_followed():
    """Offsets that are not a run's: nothing outside the matrices is read or written, what is inside may be anything."""
    guard = torch.full((40, 8), 7.0, device="cuda")
    op = ExpertProduct(6, 8, 8, 3, dtype=torch.float32)
    for start in ([0, 1000, 2000, 3000], [-5, 2, 4, 6], [0, 6, 3, 1 << 40]):
        X = torch.ones(6, 8, device="cuda")
        Y = guard.clone()
        B.regot_expert_product(X, torch.ones(3, 8, 8, device="cuda"), torch.tensor(start, device="cuda"), Y[10:16])
        assert bool((Y[:10] == 7.0).all()) and bool((Y[16:] == 7.0).all())
        op.weight_grad(X, X, torch.tensor(start, device="cuda"))
    order = torch.tensor([0, 5, -1, 2 ** 31 - 1, 100, -2 ** 31], dtype=torch.int32, device="cuda")
    op.product(torch.ones(3, 8, device="cuda"), torch.ones(3, 8, 8, device="cuda"), torch.tensor([0, 2, 4, 6], device="cuda"), order, 2)
    assert bool((op.Y == 8.0).all())


def test_gradients_against_differences():
    """32 bits: Y is linear in X and in W, so a difference of two calls has no error but its roundings."""
    c = Case(50, 2, 5, 40, 24, torch.float32)
    start, order, k = c.on()
    g = matrix(c.gen, c.rows, c.m, torch.float32)
    op = c.op()
    op.input_grad(g, c.W, start)
    op.weight_grad(g, c.X, start, order, k)

    def total(X, W):
        op.product(X, W, start, order, k)
        return float((op.Y[:c.live].double() * g[:c.live].double()).sum())

    size = float((g.double().abs().sum() * 4)) * (c.d + 16) * 2.0 ** -23
    step = matrix(c.gen, c.n, c.d, torch.float32)
    source = (c.order[:c.live].long() // k).cuda()
    want = float((op.dX[:c.live].double() * step[source].double()).sum())
    assert abs((total(c.X + step, c.W) - total(c.X - step, c.W)) / 2 - want) < size
    step = weights(c.gen, c.experts, c.m, c.d, torch.float32)
    want = float((op.dW.double() * step.double()).sum())
    assert abs((total(c.X, c.W + step) - total(c.X, c.W - step)) / 2 - want) < size


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
def test_the_same_call_gives_the_same_bits(dtype):
    c = Case(700, 2, 6, 200, 136, dtype, gated=True)
    op = c.op()
    dZ = matrix(c.gen, c.rows, c.wide, dtype)
    runs = []
    for _ in range(3):
        op.product(c.X, c.W, *c.on())
        op.input_grad(dZ, c.W, c.start.cuda())
        op.weight_grad(dZ, c.X, *c.on())
        runs.append([t[:c.live].clone() for t in (op.Y, op.saved, op.dX)] + [op.dW.clone()])
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))
