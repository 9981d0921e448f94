"""Builds libfairserve.so for gfx950 with hipcc (in-tree, next to this file)."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libfairserve.so")
SOURCES = ["fs_api.hip", "fs_cost.hip", "fs_history.hip", "fs_throttle.hip", "fs_sched.hip",
           "fs_sched_onchip.hip", "fs_metrics.hip", "fs_workload.hip", "fs_engine_api.hip",
           "fs_linear.hip", "fs_rope.hip", "fs_attention.hip", "fs_sample.hip", "fs_cache_api.hip",
           "fs_append4.hip", "fs_attention4.hip", "fs_pages.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # no packed fp32 instructions anywhere in device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-munsafe-fp-atomics", "-Wall", "-Wno-unused-function",
]


def build(verbose: bool = False) -> str:
    tmp = LIB + ".tmp"

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)

    # one compiler for each source, at most eight at a time (a few hundred MB each)
    with tempfile.TemporaryDirectory() as out, ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        objs = [os.path.join(out, s[:-4] + ".o") for s in SOURCES]
        list(pool.map(run, ([HIPCC, *FLAGS, "-c", os.path.join(CSRC, s), "-o", o]
                            for s, o in zip(SOURCES, objs))))
        run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    build(verbose="-v" in sys.argv)
    print(LIB)
