"""Compile the HIP library in-tree: paper_2605_08793_amd/libregot.so (gfx950 only)."""
import concurrent.futures
import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SRCS = [os.path.join(HERE, "csrc", "regot.hip"), os.path.join(HERE, "csrc", "regot_pattern.hip"),
        os.path.join(HERE, "csrc", "regot_rows.hip")]
LIB = os.path.join(HERE, "libregot.so")

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "csrc"),
    # keep the compiler from forming packed-fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wextra", "-Wno-unused-parameter",
]


def build(verbose: bool = False, extra=()) -> str:
    """Each source on its own, at the same time, then the library of their objects."""
    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)

    with tempfile.TemporaryDirectory() as objects, concurrent.futures.ThreadPoolExecutor(len(SRCS)) as pool:
        made = [os.path.join(objects, os.path.basename(src) + ".o") for src in SRCS]
        list(pool.map(lambda pair: run(["hipcc", *HIPCC_FLAGS, *extra, "-c", pair[0], "-o", pair[1]]), zip(SRCS, made)))
        run(["hipcc", "--offload-arch=gfx950", "-fPIC", "-shared", *made, "-o", LIB])
    return LIB


if __name__ == "__main__":
    print(build(verbose=True, extra=sys.argv[1:]))
