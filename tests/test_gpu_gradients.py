"""The norm over many tensors, and clipping, against plain 64-bit arithmetic."""
import math

import pytest
import torch

from paper_2605_08793_amd import binding as B
from paper_2605_08793_amd.experts import GradClip
from rows_reference import HALF_UNIT, TYPES, TYPE_IDS, U

pytestmark = pytest.mark.gpu


def norm_of(tensors):
    return math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in tensors))


def check(tensors, out, max_norm):
    """norm: fp64, rounded once.  factor: the same.  A number: factor's rounding, the product's, and its type's half unit."""
    want = norm_of(tensors)
    before = [t.clone() for t in tensors]
    op = GradClip(tensors, out=out)
    op.norm()
    assert abs(float(op.norm_out) - want) <= want * (U + 1e-12)
    op.clip(max_norm)
    assert abs(float(op.norm_out) - want) <= want * (U + 1e-12)
    factor = max_norm / want if want > max_norm else 1.0
    assert abs(float(op.factor) - factor) <= factor * (U + 1e-12)
    for t, b, o in zip(tensors, before, tensors if out is None else out):
        rel, least = HALF_UNIT[t.dtype]
        x = b.double() * factor
        assert bool(((o.double() - x).abs() <= x.abs() * (2.1 * U + rel * (1 + 1e-6)) + least).all())
        if out is not None:
            assert torch.equal(t, b)


SIZES = [[1], [0], [7], [0, 3, 0, 2049], [2047, 2048, 2049, 5000], [1] * 250, [100000, 1, 65536, 33], [3_000_001], [17_000_000, 12], [40000] * 101]


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{s[0]}")
def test_norm_and_clip(sizes, dtype):
    gen = torch.Generator(device="cuda").manual_seed(len(sizes))
    tensors = [torch.randn(s, generator=gen, device="cuda").to(dtype) for s in sizes]
    whole = max(norm_of(tensors), 1.0)
    for limit in (0.37, 5.0):
        check([t.clone() for t in tensors], None, limit * whole)
        check(tensors, [torch.full_like(t, 3.0) for t in tensors], limit * whole)


def test_types_together_and_odd_addresses():
    gen = torch.Generator(device="cuda").manual_seed(1)
    wide = [torch.randn(9000, generator=gen, device="cuda").to(t) for t in TYPES]
    tensors = [w[a:b] for w in wide for a, b in ((1, 4), (5, 2060), (2061, 8999))] + [torch.randn(3, 5, 7, generator=gen, device="cuda")]
    gaps = [w[[0, 4, 2060, 8999]].clone() for w in wide]
    check(tensors, None, 0.5)
    for w, g in zip(wide, gaps):
        assert torch.equal(w[[0, 4, 2060, 8999]], g)


def test_numbers_whose_squares_are_beyond_32_bits():
    t = torch.tensor([3e30, 4e30], device="cuda")
    op = GradClip([t, torch.full((4,), 1e-30, device="cuda")])
    op.clip(1.0)
    assert abs(float(op.norm_out) - 5e30) < 5e30 * 2 * U
    assert torch.allclose(t, torch.tensor([0.6, 0.8], device="cuda"), rtol=4 * U)
    small = torch.tensor([3e-30, 4e-30], device="cuda")
    op = GradClip([small])
    op.norm()
    assert abs(float(op.norm_out) - 5e-30) < 5e-30 * 2 * U


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("count", [10, 3_000_000])
def test_a_norm_that_is_not_finite_scales_nothing(bad, count):
    t = torch.ones(count, device="cuda")
    t[count // 2] = bad
    before = t.clone()
    out = torch.zeros_like(t)
    op = GradClip([t], out=[out])
    op.clip(0.5)
    assert not math.isfinite(float(op.norm_out)) and float(op.factor) == 1.0
    assert torch.equal(out.nan_to_num(nan=123.0), before.nan_to_num(nan=123.0))
    GradClip([t]).clip(0.5)
    assert torch.equal(t.nan_to_num(nan=123.0), before.nan_to_num(nan=123.0))


def test_a_limit_that_is_not_reached_leaves_everything():
    t = torch.randn(5000, device="cuda")
    before = t.clone()
    op = GradClip([t])
    for limit in (float("inf"), 1e30, float(t.double().norm()) * (1 + 1e-6)):
        op.clip(limit)
        assert float(op.factor) == 1.0 and torch.equal(t, before)


def test_no_tensors():
    op = GradClip([])
    op.clip(1.0)
    assert float(op.norm_out) == 0.0 and float(op.factor) == 1.0


def test_refusals():
    a = torch.zeros(100, device="cuda")
    for tensors, out in (([a, a], None), ([a[:60], a[50:]], None), ([a[:50]], [a[25:75]]), ([a[:50], a[50:]], [a[50:], torch.zeros(50, device="cuda")])):
        with pytest.raises(B.RegotError):
            GradClip(tensors, out=out).clip(1.0)
    GradClip([a[:60], a[50:]]).norm()      # (reading twice is fine)
    for limit in (0.0, -1.0, float("nan")):
        with pytest.raises(B.RegotError):
            GradClip([a]).clip(limit)
    for bad in ([a.double()], [a[::2]], [a.cpu()], ["a"]):
        with pytest.raises(TypeError):
            GradClip(bad)
    for bad in ([torch.zeros(99, device="cuda")], [a.half()], []):
        with pytest.raises(TypeError):
            GradClip([a], out=bad)
