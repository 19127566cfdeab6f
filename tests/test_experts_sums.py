"""The sums of the 16-bit products, which assembly statements add up in the accumulation registers, in the code that the compiler makes of this source: from the first product to the
wait behind the last, nothing but products touches these registers (the compiler does not know how long a product takes, so a sum that it copied or moved away there
would be read too early).  Compiled for the GPU, without one."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2605_08793_amd import build

SOURCE = os.path.join(build.HERE, "csrc", "regot_experts_{}.hip")


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_sums_stay_where_they_are(tmp_path):
    types = ["bf16", "f16"]
    running = [subprocess.Popen(["hipcc", *build.HIPCC_FLAGS, "-w", "-S", "--cuda-device-only", SOURCE.format(t), "-o", str(tmp_path / f"{t}.s")], stdout=subprocess.DEVNULL,
                                stderr=subprocess.DEVNULL) for t in types]
    assert [p.wait(timeout=400) for p in running] == [0, 0]
    for t in types:
        products, waits, wrong, kernels = 0, 0, [], 0
        kernel, busy, by_hand = None, False, False
        for line in (tmp_path / f"{t}.s").read_text().split("\n"):
            if re.match(r"_ZN5regot\w*expert_tile_kernel\w*:", line):
                kernel, busy, kernels = line, False, kernels + 1
            elif ".Lfunc_end" in line:
                assert not busy, f"{kernel}: no wait behind the last product"
                kernel = None
            elif "#ASMSTART" in line or "#ASMEND" in line:
                by_hand = "#ASMSTART" in line
            elif kernel and by_hand and "v_mfma" in line:
                busy, products = True, products + 1
            elif kernel and by_hand and "s_nop 15" in line:
                busy, waits = False, waits + 1
            elif busy and re.search(r"\ba(\d|\[\d)", line.split(";")[0]):
                wrong.append((kernel, line))
        assert not wrong, wrong[:5]
        assert kernels > 10 and products >= 40 * kernels // 2 and waits >= kernels // 2, (kernels, products, waits)
