"""Alternatives of long rows whose best columns are more than the threads' maxima tell apart: equal scores, and few open columns."""
import numpy as np
import pytest
import torch

from rows_reference import TYPE_IDS, TYPES
from test_gpu_rows_logprob import call, check, scores
from test_gpu_rows_many_alternatives import time

pytestmark = pytest.mark.gpu


def rows(kind, n, m, dtype):
    S = scores(n, m, dtype, m)
    if kind == "equal":
        S[:] = -1.5
    elif kind == "two values":
        S = (S > 0).to(dtype)
    elif kind.startswith("run of"):
        count = int(kind.split()[-1])
        begin = m // 3
        S[:, :begin] = -np.inf
        S[:, begin + count:] = -np.inf
    elif kind == "few places":  # open columns of ten threads only, in all stretches of the row
        S[:, torch.arange(m) % 2048 >= 80] = -np.inf
    elif kind == "few places, equal":
        S[:] = -np.inf
        S[:, torch.arange(m) % 2048 < 80] = 0.5
    return S


@pytest.mark.parametrize("kind", ["equal", "two values", "run of 130", "run of 520", "run of 800", "run of 1020", "run of 2100", "few places",
                                  "few places, equal"])
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("n,m", [(3, 4101), (250, 9000), (3, 66000), (2, 131072)])
def test_the_columns(kind, dtype, n, m):
    S = rows(kind, n, m, dtype)
    for k in (9, 60, 65, 66, 100, 127, 128):
        check(call(S.cuda(), None, 1.0, k), S, None, 1.0, k, None, f"{kind} {n}x{m} k={k}")


@pytest.mark.parametrize("n,m", [(256, 131072), (4, 131072), (512, 20000)])
@pytest.mark.parametrize("kind", ["equal", "run of 800"])
def test_no_pass_for_each_alternative(n, m, kind):
    """One by one took 25 to 180 times as long as ordinary scores (256 x 131072 34 us); with the wide list it is 3 to 11 times."""
    ordinary, S = (rows(k, n, m, torch.bfloat16).cuda() for k in ("ordinary", kind))
    assert time(S, 100) < 18 * time(ordinary, 100)
