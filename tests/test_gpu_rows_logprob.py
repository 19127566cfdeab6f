"""Log probabilities, entropy, alternatives and their gradient against plain 64-bit ones; bounds in rows_reference."""
import numpy as np
import pytest
import torch

import rows_reference as ref
from paper_2605_08793_amd import binding as B
from paper_2605_08793_amd.rows import RowLogprob
from rows_reference import TYPE_IDS, TYPES, close

pytestmark = pytest.mark.gpu


def scores(n, m, dtype, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(n, m, generator=g) * spread).to(dtype)


def laid_out(S, ld, offset, fill=float("nan")):
    """S on the GPU with rows `ld` apart, starting `offset` elements into its memory; what lies between is `fill`."""
    n, m = S.shape
    flat = torch.full((offset + n * ld + 64,), fill, dtype=S.dtype, device="cuda")
    view = flat[offset:offset + n * ld].view(n, ld)[:, :m]
    view.copy_(S)
    return flat, view


def call(S, target, eta, k, bias=None):
    n, m = S.shape
    op = RowLogprob(n, m, k=k, targets=0 if target is None else target.shape[1], dtype=S.dtype)
    for t in (op.logprob_out, op.entropy, op.stats, op.top_logprob):
        if t is not None:
            t.fill_(12345.0)
    if k:
        op.top_idx.fill_(-7)
    op.logprob(S, target, eta=eta, bias=bias)
    torch.cuda.synchronize()
    return op


def check(op, S, target, eta, k, bias, what):
    R = ref.Rows(S, bias, eta)
    bad, none = R.bad, R.none
    n, m = R.x.shape
    mx, L, H = R.max.clone(), torch.where(none, -np.inf, R.L), R.H.clone()
    mx[bad], L[bad], H[bad] = np.nan, np.nan, np.nan
    close(op.stats[:, 0], mx, 0.0, what + " max")
    close(op.stats[:, 1], L, R.tol_L, what + " log-sum")
    close(op.entropy, H, R.tol_H, what + " entropy")
    if target is not None:
        t = target.cpu().long()
        ok = (t >= 0) & (t < m)
        if m:
            at = t.clamp(0, m - 1)
            want, tol = R.logp.gather(1, at), R.tol_logp.gather(1, at)
        else:
            want = tol = torch.zeros(t.shape, dtype=torch.float64)
        want = torch.where(none[:, None], -np.inf, want)
        want = torch.where(bad[:, None], np.nan, want)
        close(op.logprob_out, torch.where(ok, want, 0.0), tol, what + " logprob")
    if k:
        idx, val = ref.best(torch.where(bad[:, None], -np.inf, R.x), k)
        idx[bad] = -1
        assert torch.equal(op.top_idx.cpu().long(), idx), what + " alternatives"
        if m:
            at = idx.clamp(0, m - 1)
            want, tol = R.logp.gather(1, at), R.tol_logp.gather(1, at)
        else:
            want = tol = torch.zeros(idx.shape, dtype=torch.float64)
        want = torch.where(idx < 0, -np.inf, want)
        close(op.top_logprob, torch.where(bad[:, None], np.nan, want), tol, what + " alternatives' logprob")


def targets_for(n, m, count, seed):
    g = torch.Generator().manual_seed(seed + 99)
    t = torch.randint(0, max(m, 1), (n, count), generator=g, dtype=torch.int32)
    if n > 1:
        t[1, 0] = -1
    if n > 2:
        t[2, -1] = m
    return t.cuda()


SIZES = [(1, 1, 1), (3, 2, 5), (5, 7, 3), (64, 63, 8), (17, 64, 64), (3, 65, 1), (2, 257, 20), (129, 1000, 10), (40, 2049, 128),
         (9, 4097, 33), (300, 3001, 5), (7, 16385, 20), (3, 70001, 64), (1, 131072, 20), (2, 200003, 128), (2500, 129, 4),
         (97, 53300, 20), (193, 53300, 9), (5, 600001, 40), (130, 4096, 50)]


@pytest.mark.parametrize("n,m,k", SIZES)
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
def test_sizes(n, m, k, dtype):
    S = scores(n, m, dtype, n * 7 + m)
    target = targets_for(n, m, 2, m)
    op = call(S.cuda(), target, 0.8, k)
    check(op, S, target, 0.8, k, None, f"{n}x{m}")


@pytest.mark.parametrize("offset,extra", [(0, 0), (1, 0), (3, 1), (8, 8), (5, 13)])
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
def test_rows_that_start_anywhere(offset, extra, dtype):
    for n, m in ((4, 5003), (33, 301), (6, 9)):
        S = scores(n, m, dtype, offset + m)
        bias = torch.randn(m, generator=torch.Generator().manual_seed(1))
        flat, view = laid_out(S, m + extra, offset)
        target = targets_for(n, m, 1, m)
        op = call(view, target, 1.0, 7, bias.cuda())
        check(op, S, target, 1.0, 7, bias, f"{n}x{m} at {offset}+{extra}")


def masked(kind, dtype, n, m):
    S = scores(n, m, dtype, 5)
    lowest = torch.finfo(dtype).min
    if kind == "third":
        S[:, torch.rand(m, generator=torch.Generator().manual_seed(2)) < 0.4] = -np.inf
    elif kind == "one left":
        S[:] = -np.inf
        S[torch.arange(n), torch.arange(n) * 37 % m] = 1.5
    elif kind == "rows of nothing":
        S[::2] = -np.inf
    elif kind == "lowest":
        S[:, ::3] = lowest
        S[1] = lowest
    elif kind == "nan and inf":
        S[0, m - 1] = np.nan
        S[1, m // 2] = np.inf
        S[2] = -np.inf
        S[2, 3] = np.nan
        S[3, 0] = -np.inf
    elif kind == "constant":
        S[:] = 0.25
    elif kind == "zeros of both signs":
        S[:] = 0.0
        S[:, ::2] = -0.0
    elif kind == "ascending":
        S[:] = torch.linspace(-5, 5, m).to(dtype)
    elif kind == "descending":
        S[:] = torch.linspace(5, -5, m).to(dtype)
    elif kind == "two values":
        S[:] = (torch.rand(n, m, generator=torch.Generator().manual_seed(3)) < 0.5).to(dtype)
    elif kind == "one far above":
        S[:, m // 3] = 300.0
    elif kind == "large":
        S *= 1000.0
    elif kind == "end only":  # what is above the rest lies in the last columns
        S[:] = -2.0
        S[:, -5:] = 3.0
    return S


KINDS = ["third", "one left", "rows of nothing", "lowest", "nan and inf", "constant", "zeros of both signs", "ascending",
         "descending", "two values", "one far above", "large", "end only"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("n,m", [(6, 777), (5, 20011), (5, 66000)])
def test_masks_and_values(kind, dtype, n, m):
    S = masked(kind, dtype, n, m)
    target = targets_for(n, m, 2, 3)
    for k in (0, 20, 128):
        op = call(S.cuda(), target, 0.5, k)
        check(op, S, target, 0.5, k, None, f"{kind} {n}x{m} k={k}")


def test_fewer_open_columns_than_alternatives():
    S = torch.full((3, 5000), -np.inf)
    S[0, [17, 4999]] = torch.tensor([1.0, 2.0])
    S[1, :3] = 0.0
    op = call(S.cuda(), None, 1.0, 10)
    check(op, S, None, 1.0, 10, None, "few open")
    assert op.top_idx[0].tolist() == [4999, 17] + [-1] * 8


def test_no_columns_and_no_rows():
    S = torch.empty(4, 0, device="cuda")
    target = torch.zeros(4, 1, dtype=torch.int32, device="cuda")
    op = call(S, target, 1.0, 3)
    check(op, S.cpu(), target, 1.0, 3, None, "no columns")
    op = RowLogprob(0, 10, k=2, targets=1, dtype=torch.float32)
    op.logprob(torch.empty(0, 10, device="cuda"), torch.empty(0, 1, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()


def test_bias_of_minus_infinity_closes_a_column():
    S = scores(5, 3000, torch.bfloat16, 1)
    bias = torch.zeros(3000)
    bias[::2] = -np.inf
    op = call(S.cuda(), None, 1.0, 30, bias.cuda())
    check(op, S, None, 1.0, 30, bias, "closed by the bias")
    assert (op.top_idx % 2 == 1).all()


def test_offsets_beyond_32_bits():
    n, m, ld = 4, 1031, 1_500_000_000
    flat = torch.empty((n - 1) * ld + m, dtype=torch.bfloat16, device="cuda")
    view = flat.as_strided((n, m), (ld, 1))
    S = scores(n, m, torch.bfloat16, 8)
    view.copy_(S)
    target = targets_for(n, m, 1, 0)
    op = call(view, target, 1.0, 9)
    check(op, S, target, 1.0, 9, None, "far rows")
    g = torch.ones(n, 1, device="cuda")
    out = op.grad(view, target, g)
    want, tol = ref.logprob_grad(ref.Rows(S, None, 1.0), target, g, None)
    close(out, want, ref.rounded(want, tol, torch.bfloat16), "far rows, gradient")


def test_many_rows():
    n, m = 300_000, 9
    S = scores(n, m, torch.float32, 4)
    target = targets_for(n, m, 1, 4)
    op = call(S.cuda(), target, 1.0, 2)
    check(op, S, target, 1.0, 2, None, "many rows")


def test_same_bits_every_time():
    for n, m in ((1, 131072), (70, 20000), (5000, 300)):
        S = scores(n, m, torch.bfloat16, 2).cuda()
        target = targets_for(n, m, 1, 2)
        first = call(S, target, 0.9, 20)
        for _ in range(3):
            again = call(S, target, 0.9, 20)
            for a, b in ((first.logprob_out, again.logprob_out), (first.entropy, again.entropy), (first.stats, again.stats),
                         (first.top_idx, again.top_idx), (first.top_logprob, again.top_logprob)):
                assert torch.equal(a, b)


def test_the_parts_that_are_left_out():
    S = scores(6, 5000, torch.float16, 6)
    full = call(S.cuda(), targets_for(6, 5000, 2, 1), 1.0, 5)
    ws = full.workspace
    lp = torch.empty(6, 2, device="cuda")
    B.regot_row_logprob(S.cuda(), targets_for(6, 5000, 2, 1), 1.0, lp, None, None, None, None, workspace=ws)
    assert torch.equal(lp, full.logprob_out)
    stats = torch.empty(6, 2, device="cuda")
    B.regot_row_logprob(S.cuda(), None, 1.0, None, None, stats, None, None, workspace=ws)
    assert torch.equal(stats, full.stats)


# ---- gradient ----------------------------------------------------------------------------------------------------------

def gradient(S, target, eta, bias, g, h, extra=0, offset=0):
    n, m = S.shape
    op = call(S.cuda(), target, eta, 0, None if bias is None else bias.cuda())
    flat = torch.full((offset + n * (m + extra) + 64,), 7.0, dtype=S.dtype, device="cuda")
    dS = flat[offset:offset + n * (m + extra)].view(n, m + extra)[:, :m]
    B.regot_row_logprob_grad(S.cuda(), target, eta, op.stats, op.entropy if h is not None else None, g, h, dS,
                             bias=None if bias is None else bias.cuda())
    torch.cuda.synchronize()
    out = dS.cpu()
    dS.fill_(7.0)
    assert bool((flat == 7.0).all()), "written outside the rows"
    return out


@pytest.mark.parametrize("n,m", [(1, 1), (3, 2), (9, 63), (33, 1000), (700, 129), (5, 4097), (300, 3001), (3, 70001), (2, 131072)])
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
def test_gradient(n, m, dtype):
    S = scores(n, m, dtype, m + n)
    R_bias = torch.randn(m, generator=torch.Generator().manual_seed(m)) if m % 2 else None
    g = torch.randn(n, 3, generator=torch.Generator().manual_seed(1)).cuda()
    h = torch.randn(n, generator=torch.Generator().manual_seed(2)).cuda()
    target = targets_for(n, m, 3, n)
    if m > 8:
        target[0, 1] = target[0, 0]  # the same column twice
    R = ref.Rows(S, R_bias, 0.6)
    for gg, hh, tt, extra, offset in ((g, h, target, 0, 0), (g, None, target, 3, 1), (None, h, None, 1, 5)):
        want, tol = ref.logprob_grad(R, tt, gg, hh)
        close(gradient(S, tt, 0.6, R_bias, gg, hh, extra, offset), want, ref.rounded(want, tol, dtype), f"{n}x{m} {extra}+{offset}")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
def test_gradient_of_masked_rows(kind, dtype):
    n, m = 6, 5011
    S = masked(kind, dtype, n, m)
    g, h = torch.full((n, 2), 0.5).cuda(), torch.full((n,), -0.3).cuda()
    target = targets_for(n, m, 2, 3)
    R = ref.Rows(S, None, 0.5)
    want, tol = ref.logprob_grad(R, target, g, h)
    close(gradient(S, target, 0.5, None, g, h), want, ref.rounded(want, tol, dtype), kind)


def test_gradient_against_differences():
    n, m, eta = 4, 900, 0.7
    S = scores(n, m, torch.float32, 12)
    target = targets_for(n, m, 2, 3)
    g, h = torch.randn(n, 2, generator=torch.Generator().manual_seed(3)).cuda(), torch.randn(n, generator=torch.Generator().manual_seed(4)).cuda()
    out = gradient(S, target, eta, None, g, h).double()

    def value(x):
        lp = torch.log_softmax(x / eta, 1)
        t = target.cpu().long()
        ok = (t >= 0) & (t < m)
        return float((g.cpu().double() * torch.where(ok, lp.gather(1, t.clamp(0, m - 1)), 0.0)).sum() - (h.cpu().double() * (lp.exp() * lp).sum(1)).sum())

    rng = torch.Generator().manual_seed(5)
    for _ in range(5):
        v = torch.randn(n, m, generator=rng, dtype=torch.float64)
        # central differences: the error is (step^2 / 6) times a third derivative of the order of |v|^3 sums, and 1e-16 / step of rounding
        step = 1e-4
        slope = (value(S.double() + step * v) - value(S.double() - step * v)) / (2 * step)
        _, tol = ref.logprob_grad(ref.Rows(S, None, eta), target, g, h)
        bound = float((ref.rounded(out, tol, torch.float32) * v.abs()).sum()) + 1e-5
        assert abs(float((out * v).sum()) - slope) <= bound


def test_on_a_stream_of_its_own():
    S = scores(50, 20000, torch.bfloat16, 3).cuda()
    target = targets_for(50, 20000, 1, 3)
    want = call(S, target, 1.0, 5)
    op = RowLogprob(50, 20000, k=5, targets=1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        op.logprob(S, target)
    side.synchronize()
    assert torch.equal(op.logprob_out, want.logprob_out) and torch.equal(op.top_idx, want.top_idx)
