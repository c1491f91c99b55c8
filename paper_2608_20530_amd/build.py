"""Build the HIP library liblilicorr.so in-tree for gfx950 (hipcc, no torch extension)."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liblilicorr.so")
# measurement aid for bench.py (a plain streaming read), kept out of the path's library
BENCH_LIB = os.path.join(HERE, "libbench_read.so")
SOURCES = ["topk.hip", "vectors.hip", "pairs.hip", "walk.hip", "viterbi.hip", "fused.hip",
           "graph.hip", "scorer.hip", "paged.hip", "attention.hip", "attention4.hip",
           "evict.hip", "status.hip"]

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    # packed fp32 VALU instructions stay disabled (wrong results seen on this hardware class)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument",
]


def _hipcc(out: str, sources: list[str], verbose: bool) -> None:
    cmd = ["hipcc", *FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-o", out + ".tmp", *[os.path.join(CSRC, s) for s in sources]]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    os.replace(out + ".tmp", out)


def build(verbose: bool = False) -> str:
    _hipcc(LIB, SOURCES, verbose)
    _hipcc(BENCH_LIB, ["bench_read.hip"], verbose)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
