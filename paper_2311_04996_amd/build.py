"""Build step: compiles the HIP decoder for gfx950 into libwfstdec.so next to this file."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(_HERE)
LIB_PATH = os.path.join(_HERE, "libwfstdec.so")
SOURCES = [os.path.join(_HERE, "csrc", "wfst_decoder.hip")]
# the operators beside the decoder, in the same library
OUTPUT_SOURCES = [os.path.join(_HERE, "csrc", "wfst_outputs.hip")]
HEADERS = [os.path.join(ROOT, "include", "wfst_decoder.h")]
# measured ceilings of the chip (copy, random lines, atomics): a library of its own, used by bench.py
PROBE_LIB_PATH = os.path.join(_HERE, "libwfstprobe.so")
PROBE_SOURCES = [os.path.join(_HERE, "csrc", "wfst_probe.hip")]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-std=c++17", "-fPIC",
    "-ffp-contract=off",                       # costs are compared bit for bit: no FMA contraction
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I" + os.path.join(ROOT, "include"),
]


def build_library(verbose: bool = False) -> str:
    """Always recompiles both libraries.  Returns the path of the decoder's shared library."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.check_call(cmd, stderr=None if verbose else subprocess.DEVNULL)

    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(3) as pool:
        # The decoder is optimised for size: its frame loop is about 70 KB of code, more than the
        # instruction cache holds, and the smaller build measured 2 % faster than -O3 (-O2 1 %, -Oz slower).
        objects = [(src, opt, os.path.join(tmp, os.path.basename(src) + ".o"))
                   for srcs, opt in ((SOURCES, "-Os"), (OUTPUT_SOURCES, "-O3")) for src in srcs]
        jobs = [pool.submit(run, [hipcc, opt] + HIPCC_FLAGS + ["-c", "-o", obj, src]) for src, opt, obj in objects]
        jobs.append(pool.submit(run, [hipcc, "-O3", "-shared"] + HIPCC_FLAGS + ["-o", PROBE_LIB_PATH] + PROBE_SOURCES))
        for j in jobs:
            j.result()
        run([hipcc, "--offload-arch=gfx950", "-fPIC", "-shared", "-o", LIB_PATH] + [obj for _, _, obj in objects])
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(verbose=True))
