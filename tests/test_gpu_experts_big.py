"""Products grouped by expert in tiles of 256 x 256, which calls of many tiles take: products of few experts with several tiles and a part of one and many columns;
weight gradients of many experts, some with several stretches, most with a few rows or none; and products of those in smaller tiles."""
import pytest
import torch

import experts_reference as ref
from paper_2605_08793_amd.experts import ExpertProduct
from rows_reference import U
from test_gpu_experts_product import Case, matrix, same_beyond

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]


def uneven(n, k, experts, gen):
    """Most choices to three experts, whose runs then are several tiles and a part of one, the others anywhere; of few experts, about evenly."""
    idx = torch.randint(0, experts, (n, k), generator=gen)
    if experts < 8:
        idx[torch.rand(n, k, generator=gen) < 0.05] = -1
        return idx.to(torch.int32)
    idx[torch.rand(n, k, generator=gen) < 0.8] = 5
    idx[torch.rand(n, k, generator=gen) < 0.3] = experts - 1
    idx[torch.rand(n, k, generator=gen) < 0.1] = 6
    idx[torch.rand(n, k, generator=gen) < 0.05] = -1
    return idx.to(torch.int32)


def case(n, k, experts, d, m, dtype, **kw):
    c = Case(n, k, experts, d, m, dtype, **kw)
    c.start, c.order, c.place = ref.order(uneven(n, k, experts, c.gen), experts)
    c.live = int(c.start[-1])
    return c


SIZES = [(900, 2, 1024, 64, 8), (700, 2, 520, 8, 304), (1500, 1, 1024, 200, 128), (400, 4, 600, 136, 264), (1300, 2, 4, 72, 13000), (1100, 1, 3, 8, 29960), (2100, 1, 1, 200, 15008),
         (1300, 2, 4, 72, 14344), (1100, 1, 3, 8, 34952)]


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("turned", [False, True], ids=["outputs", "inputs"])
@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
@pytest.mark.parametrize("n,k,experts,d,m", SIZES)
def test_product(n, k, experts, d, m, gated, turned, dtype):
    c = case(n, k, experts, d, m, dtype, turned=turned, gated=gated, gap=8)
    op = c.op()
    op.product(c.X, c.W, *c.on())
    z, tol = ref.sums(c.wide_rows(), c.W.cpu().double(), c.start)
    h, t = ref.gate(z, tol) if gated else (z, tol)
    ref.close(op.Y[:c.live], h[:c.live], ref.rounded(h, t, dtype)[:c.live], "Y")
    same_beyond(op.Y, c.live)
    if gated:
        ref.close(op.saved[:c.live], z[:c.live], ref.rounded(z, tol, dtype)[:c.live], "saved")
        same_beyond(op.saved, c.live)
        without = ExpertProduct(c.rows, m, d, experts, gated=True, dtype=dtype)
        without.product(c.X, c.W, *c.on())
        assert torch.equal(without.Y[:c.live], op.Y[:c.live])


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("behind_gate", [False, True], ids=["plain", "behind gate"])
@pytest.mark.parametrize("turned", [False, True], ids=["outputs", "inputs"])
@pytest.mark.parametrize("n,k,experts,d,m", [(n, k, e, m, d) for n, k, e, d, m in SIZES])
def test_gradients(n, k, experts, d, m, turned, behind_gate, dtype):
    c = case(n, k, experts, d, m, dtype, turned=turned)
    start, order, k = c.on()
    dY = matrix(c.gen, c.rows, m, dtype, 8)
    op = c.op()
    D, tol = ref.sums(dY.cpu().double(), c.W.cpu().double().transpose(1, 2), c.start)
    op.dX = torch.full((c.rows, 2 * d if behind_gate else d), 7.0, dtype=dtype, device="cuda")
    if behind_gate:
        saved = matrix(c.gen, c.rows, 2 * d, dtype, 8, scale=3.0)
        op.input_grad(dY, c.W, start, saved=saved)
        D, tol = ref.gate_grad(D, tol, saved.cpu().double())
    else:
        op.input_grad(dY, c.W, start)
    ref.close(op.dX[:c.live], D[:c.live], ref.rounded(D, tol, dtype)[:c.live], "dX")
    same_beyond(op.dX, c.live)
    for gather in (True, False):
        X = c.X if gather else matrix(c.gen, c.rows, d, dtype, 8)
        want, tol = ref.weight_grad(dY.cpu().double(), c.wide_rows() if gather else X.cpu().double(), c.start)
        for out in (dtype, torch.float32):
            op = c.op(grad_dtype=out)
            op.weight_grad(dY, X, start, order if gather else None, k if gather else 1)
            ref.close(op.dW, want, ref.rounded(want, tol, out), f"dW {out} {gather}")


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("turned", [False, True], ids=["outputs", "inputs"])
def test_long_sums_behind_the_gate(turned, dtype):
    """Few rows, very many columns, so that a long sum's tiles are many.  The plain side on the device, in 64 bits."""
    rows, experts, d, m = 700, 2, 87304, 2056
    gen = torch.Generator(device="cuda").manual_seed(11)
    normal = lambda *shape, scale=1.0: (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)  # noqa: E731
    runs = [3, 300, 650]
    dY, saved = normal(rows, m), normal(rows, 2 * d, scale=3.0)
    W = normal(experts, d, m, scale=m ** -0.5).transpose(1, 2) if turned else normal(experts, m, d, scale=m ** -0.5)
    op = ExpertProduct(rows, m, d, experts, dtype=dtype)
    op.dX = torch.full((rows, 2 * d), 7.0, dtype=dtype, device="cuda")
    op.input_grad(dY, W, torch.tensor(runs, device="cuda"), saved=saved)
    for e, (a, b) in enumerate(zip(runs, runs[1:])):
        w, g = W[e].double().contiguous(), dY[a:b].double()
        D, tol = g @ w, (g.abs() @ w.abs()) * 2 * U * (m + 16) + ref.TINY
        want, tol = ref.gate_grad(D, tol, saved[a:b].double())
        ref.close(op.dX[a:b], want.cpu(), ref.rounded(want.cpu(), tol.cpu(), dtype), f"expert {e}")
    assert bool((op.dX[:3] == 7.0).all()) and bool((op.dX[650:] == 7.0).all())
