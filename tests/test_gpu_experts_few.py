"""Products grouped by expert where each has few rows: the kernel that reads the weights straight through, at the ends of its units, sums and stretches."""
import pytest
import torch

import experts_reference as ref
from test_gpu_experts_product import Case, same_beyond
from rows_reference import TYPES, TYPE_IDS

pytestmark = pytest.mark.gpu

# (n, k, experts, d, m): sums of one unit, a unit and a part of one, as many units as waves, one more, four for each wave and more; rows of W that end within
# a stretch of 32, and within a chunk of 16 bytes, many stretches; runs of 0, 1, 16, 17 and more rows
SIZES = [(1, 1, 1, 8, 8), (1, 8, 256, 2048, 96), (3, 2, 7, 64, 40), (5, 3, 4, 72, 32), (16, 1, 1, 512, 24), (17, 1, 2, 576, 1000), (40, 4, 10, 504, 264), (64, 4, 30, 2056, 72),
         (2, 1, 8, 8192, 64), (9, 8, 1024, 136, 2048),
         (12, 1, 1, 512, 24), (40, 3, 10, 504, 264), (5, 3, 4, 72, 33), (1, 8, 256, 2048, 119), (3, 2, 7, 64, 6), (40, 3, 12, 504, 1), (2, 1, 8, 8192, 59), (100, 1, 9, 4104, 150)]


@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
@pytest.mark.parametrize("gap", [0, 8])
@pytest.mark.parametrize("n,k,experts,d,m", SIZES)
def test_product(n, k, experts, d, m, gap, gated, dtype):
    c = Case(n, k, experts, d, m, dtype, gated=gated, gap=gap, dropped=0.0 if n == 1 else 0.1)
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
def test_rows_as_they_are(dtype):
    """Without an order: row r takes row r of X, of which there may be more."""
    c = Case(20, 2, 9, 256, 48, dtype)
    X = torch.randn(c.rows + 5, c.d, generator=c.gen).to(dtype).cuda()
    op = c.op()
    op.product(X, c.W, c.start.cuda())
    z, tol = ref.sums(X[:c.rows].cpu().double(), c.W.cpu().double(), c.start)
    ref.close(op.Y[:c.live], z[:c.live], ref.rounded(z, tol, dtype)[:c.live], "Y")
