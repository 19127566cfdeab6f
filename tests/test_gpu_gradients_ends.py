"""Clipping where the norm itself is beyond 32 bits, though every number is finite and the sum of squares is within 64: it is told as an infinity, and nothing is scaled."""
import math

import pytest
import torch

from paper_2605_08793_amd.experts import GradClip

pytestmark = pytest.mark.gpu

LARGEST = torch.finfo(torch.float32).max


@pytest.mark.parametrize("max_norm", [0.5, 1e38, math.inf])
@pytest.mark.parametrize("count,value", [(4, 3e38), (2, LARGEST), (3_000_000, 1e36)])
def test_a_norm_beyond_32_bits_scales_nothing(count, value, max_norm):
    """count * value^2 is above LARGEST^2 in each case; the sums of few and of many workgroups."""
    t = torch.full((count,), value, device="cuda")
    before = t.clone()
    out = torch.zeros_like(t)
    for op, to in ((GradClip([t]), t), (GradClip([t], out=[out]), out)):
        op.norm()
        assert float(op.norm_out) == math.inf
        op.clip(max_norm)
        assert float(op.norm_out) == math.inf and float(op.factor) == 1.0
        assert torch.equal(to, before)


def test_the_largest_norm_is_scaled():
    """One number: the norm is its size, and the result the limit within the roundings of norm, factor and product (2^-24 each)."""
    t = torch.tensor([-LARGEST], device="cuda")
    op = GradClip([t])
    op.clip(1e38)
    assert float(op.norm_out) == LARGEST and abs(float(op.factor) * LARGEST / 1e38 - 1) < 2.0 ** -23
    assert abs(float(t) / -1e38 - 1) < 3 * 2.0 ** -24
