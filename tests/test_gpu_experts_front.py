"""Runs that begin several tiles behind the first row, as a call on some of a layer's experts has them: rows of no run, in front and behind, are left as they were."""
import pytest
import torch

import experts_reference as ref
from paper_2605_08793_amd import binding as B
from rows_reference import TYPES, TYPE_IDS
from test_gpu_experts_product import matrix, weights

pytestmark = pytest.mark.gpu

# (rows, starts, d, m): 16 rows a tile (on average less than 12 rows an expert), one tile a row; 64 and 128 rows, whole chunks of 16 bytes and not; 256
CASES = [(90, [40, 60, 61, 61, 70, 75, 77, 79, 80], 64, 40), (7, [3, 4, 4, 5, 6, 6, 6, 6, 6], 64, 40), (1000, [300, 500, 700], 72, 40), (1000, [300, 500, 700], 33, 17),
         (2000, [700, 1500, 1900], 64, 4096), (2000, [700, 1500, 1900], 65, 4095), (2600, [800, 1500, 2500], 72, 15104)]
CASE_IDS = ["few", "row by row", "64", "64 odd", "128", "128 odd", "256"]


def filled(rows, cols, dtype):
    return torch.full((rows, cols), 7.0, dtype=dtype, device="cuda")


def check(got, want, tol, starts, what):
    ref.close(got[starts[0]:starts[-1]], want[starts[0]:starts[-1]], ref.rounded(want, tol, got.dtype)[starts[0]:starts[-1]], what)
    assert bool((got[:starts[0]] == 7.0).all()), f"{what}: rows in front of the runs were written"
    assert bool((got[starts[-1]:] == 7.0).all()), f"{what}: rows behind the runs were written"


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("turned", [False, True], ids=["outputs", "inputs"])
@pytest.mark.parametrize("rows,starts,d,m", CASES, ids=CASE_IDS)
def test_rows_in_front(rows, starts, d, m, turned, dtype):
    gen = torch.Generator().manual_seed(rows + d)
    experts, start = len(starts) - 1, torch.tensor(starts, device="cuda")
    X = matrix(gen, rows, d, dtype)
    W = weights(gen, experts, m, d, dtype, turned=turned)
    z, tol = ref.sums(X.cpu().double(), W.cpu().double(), starts)
    Y = filled(rows, m, dtype)
    B.regot_expert_product(X, W, start, Y)
    check(Y, z, tol, starts, "Y")

    if m % 2 == 0:
        Y, saved = filled(rows, m // 2, dtype), filled(rows, m, dtype)
        B.regot_expert_product(X, W, start, Y, act="gate", saved=saved)
        check(Y, *ref.gate(z, tol), starts, "gated Y")
        check(saved, z, tol, starts, "saved")

    at_gate = matrix(gen, rows, 2 * m, dtype, scale=3.0)
    Y = filled(rows, 2 * m, dtype)
    B.regot_expert_product(X, W, start, Y, act="gate_grad", saved=at_gate)
    check(Y, *ref.gate_grad(z, tol, at_gate.cpu().double()), starts, "gate's gradient")


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("rows,starts,d,m", [(120, [0, 20, 45, 46, 60, 80, 90, 100, 110], 64, 40), (1000, [0, 260, 500, 700, 990], 72, 40), (1000, [0, 260, 500, 700, 990], 33, 17)],
                         ids=["few", "64", "64 odd"])
def test_halves_of_the_experts(rows, starts, d, m, dtype):
    """Two calls, each with half of the experts, into one result: the second leaves what the first has written."""
    gen = torch.Generator().manual_seed(rows)
    experts, start = len(starts) - 1, torch.tensor(starts, device="cuda")
    half = experts // 2
    X, W = matrix(gen, rows, d, dtype), weights(gen, experts, m, d, dtype)
    z, tol = ref.sums(X.cpu().double(), W.cpu().double(), starts)
    for parts in (((0, half), (half, experts)), ((half, experts), (0, half))):
        Y = filled(rows, m, dtype)
        for a, b in parts:
            B.regot_expert_product(X, W[a:b], start[a:b + 1], Y)
        check(Y, z, tol, starts, "Y")


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("rows,starts,d,m", [(90, [40, 60, 61, 61, 70, 75, 77, 79, 80], 64, 40), (1000, [300, 500, 500, 700], 72, 40), (1000, [300, 500, 700], 33, 17), (9000, [4000, 8700], 64, 40)],
                         ids=["few", "whole", "odd", "in parts"])
def test_weight_gradients(rows, starts, d, m, dtype):
    """Rows of no run hold NaN, and slots of no token: a gradient that looked at one would be NaN."""
    gen = torch.Generator().manual_seed(rows)
    start, k = torch.tensor(starts, device="cuda"), 2
    dY, X = matrix(gen, rows, m, dtype), matrix(gen, rows, d, dtype)
    order = torch.randint(0, rows * k, (rows,), generator=gen, dtype=torch.int32)
    order[:starts[0]] = -1
    order[starts[-1]:] = -1
    for gather in (False, True):
        there = X.cpu().double()[order.long().clamp(min=0) // k] if gather else X.cpu().double()
        g, x = dY.clone(), X.clone()
        for t in (g,) if gather else (g, x):
            t[:starts[0]] = float("nan")
            t[starts[-1]:] = float("nan")
        for out in {dtype, torch.float32}:
            dW = torch.full((len(starts) - 1, m, d), 7.0, dtype=out, device="cuda")
            ws = torch.empty(B.regot_expert_weight_grad_workspace_bytes(rows, m, d, len(starts) - 1), dtype=torch.uint8, device="cuda")
            B.regot_expert_weight_grad(g, x, start, dW, order=order.cuda() if gather else None, k=k if gather else 1, workspace=ws)
            want, tol = ref.weight_grad(dY.cpu().double(), there, starts)
            ref.close(dW, want, ref.rounded(want, tol, out), f"dW {out} {gather}")
