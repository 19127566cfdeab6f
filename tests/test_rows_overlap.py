"""A gradient in the memory of its scores: shared elements are refused, rows between those of the scores are not."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import test_rows_abi as abi
from paper_2605_08793_amd import binding as B
from paper_2605_08793_amd.rows import RowDistill, RowLogprob, RowRoute

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <stdio.h>
#include <set>
#include "regot_overlap.hpp"
int main()
{
    long cases = 0, shared = 0;
    for (int b : {2, 4})
        for (int n = 0; n <= 5; ++n)
            for (int m = 0; m <= 4; ++m)
                for (int ldS = m > 0 ? m : 1; ldS <= m + 5; ++ldS)
                    for (int ldD = m > 0 ? m : 1; ldD <= m + 5; ++ldD)
                        for (int at = 0; at <= 220; at += 1) {  // bytes: unlike multiples of the element too
                            std::set<int> bytes;
                            for (int i = 0; i < n; ++i)
                                for (int j = 0; j < m * b; ++j) bytes.insert(100 + i * ldS * b + j);
                            bool want = false;
                            for (int i = 0; i < n; ++i)
                                for (int j = 0; j < m * b; ++j) want |= bytes.count(at + i * ldD * b + j) != 0;
                            if (regot::overlap(n, m, (const void *)100, ldS, (const void *)(uintptr_t)at, ldD, b) != want) {
                                printf("b %d n %d m %d ldS %d ldD %d at %d: not %d\\n", b, n, m, ldS, ldD, at, want);
                                return 1;
                            }
                            ++cases, shared += want;
                        }
    const int64_t most = 2147483647, far = (int64_t)1 << 62;
    if (!regot::overlap(most, most, (const void *)4096, far, (const void *)4096, far, 4)) return 2;
    if (regot::overlap(most, 8, (const void *)4096, 16, (const void *)(4096 + 32), 16, 4)) return 3;
    if (!regot::overlap(most, 8, (const void *)4096, 16, (const void *)(4096 + 16 * 4 * 2000000000ull), 16, 4)) return 4;
    printf("%ld cases, %ld shared\\n", cases, shared);
    return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_every_small_case(tmp_path):
    src, out = tmp_path / "overlap.cpp", tmp_path / "overlap"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2605_08793_amd", "csrc"), str(src), "-o", str(out)], check=True)
    done = subprocess.run([str(out)], capture_output=True, text=True)
    assert done.returncode == 0, (done.returncode, done.stdout)


@pytest.mark.parametrize("name", ["regot_row_logprob_grad", "regot_row_distill", "regot_row_route_grad"])
def test_shared_elements_are_refused(name):
    at = abi.P.value
    for changed in (dict(dS=abi.P), dict(dS=ctypes.c_void_p(at + 4 * 8 * 4 - 4)), dict(dS=ctypes.c_void_p(at - 4 * 8 * 4 + 4)),
                    dict(ldS=16, ldD=16, dS=ctypes.c_void_p(at + 28)), dict(ldS=16, ldD=12, dS=ctypes.c_void_p(at + 32))):
        assert abi.call(name, **changed) == abi.ARG, changed
    assert abi.call(name, n=0, dS=abi.P) == 0


@pytest.mark.gpu
def test_in_place_is_an_error_and_rows_between_are_not():
    n, m, k = 6, 5000, 4
    S = torch.randn(n, m, generator=torch.Generator().manual_seed(1)).cuda()
    idx = torch.randint(0, m, (n, k), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()
    g = torch.randn(n, k, generator=torch.Generator().manual_seed(3)).cuda()
    rows, learn, route = RowLogprob(n, m, targets=k, dtype=S.dtype), RowDistill(n, m, k, dtype=S.dtype), RowRoute(n, 100, k)
    rows.logprob(S, idx)
    want = rows.grad(S, idx, g)
    learn.distill(S, idx, g)
    route.route(S[:, :100])
    want_route = route.grad(S[:, :100], g)
    wide = torch.zeros(n, 2 * m + 100, device="cuda")
    inside, beside = wide[:, :m], wide[:, m:2 * m]
    inside.copy_(S)
    with pytest.raises(B.RegotError):
        B.regot_row_logprob_grad(inside, idx, 1.0, rows.stats, None, g, None, inside)
    with pytest.raises(B.RegotError):
        B.regot_row_distill(inside, idx, g, 1.0, learn.loss, wide[:, m - 1:2 * m - 1], workspace=learn.workspace)
    with pytest.raises(B.RegotError):
        B.regot_row_route_grad(inside[:, :100], route.idx, g, inside[:, 50:150])
    assert torch.equal(inside, S)
    B.regot_row_logprob_grad(inside, idx, 1.0, rows.stats, None, g, None, beside)
    assert torch.equal(beside, want)
    B.regot_row_distill(inside, idx, g, 1.0, learn.loss, beside, workspace=learn.workspace)
    assert torch.equal(beside, learn.grad)
    B.regot_row_route_grad(inside[:, :100], route.idx, g, inside[:, 100:200])
    assert torch.equal(inside[:, 100:200], want_route)
