"""The numbering of a grouped product's tiles, from the kernels' own header, for runs that begin and end anywhere: every row of a run is one tile's, and no tile has a row
in front of the first run, behind the last or of two experts.  On the host, without a GPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>
#include <algorithm>
#include <random>
#include <vector>
#include "regot_experts.hpp"
using namespace regot;

// the tile that the kernels give to number t: experts before it by the same rule, all of them looked at
template <int BM>
Run run_of(const std::vector<int> &start, int64_t t, bool single)
{
    const int experts = (int)start.size() - 1;
    int e = 0, s = start[0], end = 0x7fffffff;
    for (int i = 0; i < experts; ++i) {
        if (tile_is_behind<BM>(start[i + 1], i, t, single)) ++e, s = std::max(s, start[i + 1]);
        else end = std::min(end, start[i + 1]);
    }
    return e >= experts ? Run{0, 0, 0} : run_of_tile<BM>(e, s, end, t, single);
}

template <int BM>
bool right(const std::vector<int> &start, int rows)
{
    const int experts = (int)start.size() - 1;
    const bool single = rows < rows / BM + experts;
    std::vector<int> expert(rows, -1), want(rows, -1);
    for (int e = 0; e < experts; ++e)
        for (int r = start[e]; r < start[e + 1]; ++r) want[r] = e;
    for (int64_t t = 0; t < (single ? rows : rows / BM + experts); ++t) {
        const Run run = run_of<BM>(start, t, single);
        for (int64_t r = run.first; r < std::min(run.first + BM, run.end); ++r) {
            if (r < 0 || r >= rows || expert[r] != -1) return false;
            expert[r] = run.expert;
        }
    }
    return expert == want;
}

int main()
{
    std::mt19937 random(1);
    int bad = 0;
    for (int trial = 0; trial < 4000; ++trial) {
        const int rows = 1 + random() % (trial % 3 == 0 ? 40 : 3000), experts = 1 + random() % (trial % 5 == 0 ? 200 : 7);
        std::vector<int> start(experts + 1);
        for (int &s : start) s = random() % (rows + 1);
        if (trial % 2) start[0] = 0;
        std::sort(start.begin(), start.end());
        if (right<16>(start, rows) && right<64>(start, rows) && right<128>(start, rows) && right<256>(start, rows)) continue;
        if (++bad <= 5) printf("rows %d, experts %d, start[0] %d\n", rows, experts, start[0]);
    }
    printf("%d wrong\n", bad);
    return bad != 0;
}
"""


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_each_row_of_a_run_is_one_tiles(tmp_path):
    src, program = tmp_path / "numbering.hip", tmp_path / "numbering"
    src.write_text(PROGRAM)
    done = subprocess.run(["hipcc", "-std=c++17", "-O1", "--cuda-host-only", "-w", "-I", os.path.join(ROOT, "include"), "-I",
                           os.path.join(ROOT, "paper_2605_08793_amd", "csrc"), str(src), "-o", str(program)], capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
    done = subprocess.run([str(program)], capture_output=True, text=True, timeout=100)
    assert done.returncode == 0, done.stdout
