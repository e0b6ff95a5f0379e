"""Build ``libipv.so`` (HIP, gfx950) in-tree with hipcc.

Run ``python -m paper_2506_15745_amd.build`` or call :func:`build`.
"""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libipv.so")
SOURCES = [os.path.join(CSRC, "ipv_api.hip")]  # the compression pass
# the paged cache: its entry points, and the attention kernels of each page format (over rows in order, over lists of blocks)
PAGED_SOURCES = [os.path.join(CSRC, f) for f in ("ipv_paged_api.hip", "ipv_attend_bf16.hip", "ipv_attend_f32.hip",
                                                 "ipv_attend_fp8.hip", "ipv_attend_fp4.hip", "ipv_rows_api.hip",
                                                 "ipv_blocks_api.hip", "ipv_blocks_bf16.hip", "ipv_blocks_f32.hip",
                                                 "ipv_blocks_fp8.hip", "ipv_blocks_fp4.hip")]
HEADERS = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".hpp")]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
    # no packed fp32 instructions in device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("hipcc failed building libipv.so")


def build(verbose: bool = False) -> str:
    tmp = LIB + ".tmp%d" % os.getpid()
    sources = SOURCES + PAGED_SOURCES
    with tempfile.TemporaryDirectory() as folder:
        objects = [os.path.join(folder, os.path.basename(s) + ".o") for s in sources]
        with ThreadPoolExecutor(len(sources)) as pool:
            list(pool.map(lambda so: _run([HIPCC] + FLAGS + ["-c", so[0], "-o", so[1]], verbose), zip(sources, objects)))
        _run([HIPCC, "--offload-arch=gfx950", "-shared"] + objects + ["-o", tmp], verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
