"""Builds libcopyspec.so (HIP, gfx950) and nothing else.  Run as `python -m paper_2502_08923_amd.build`."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libcopyspec.so")
SOURCES = ["cs_api.hip", "cs_scan.hip", "cs_index.hip", "cs_elem.hip", "cs_gemm.hip", "cs_attn.hip",
           "cs_paged.hip", "cs_paged_attn.hip", "cs_paged_fp4.hip", "cs_paged_fp4_attn.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fno-gpu-rdc",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument"]


# The attention kernels never produce or consume a NaN (masked scores are -inf, the running
# maximum is guarded before it is subtracted), so the maxima of their softmax need no
# canonicalising copy of every operand: 18 fewer vector instructions per 32-token block.
# (Keys and values of live tokens are finite by contract; dead ones are masked before a maximum sees them.)
EXTRA_FLAGS = {"cs_attn.hip": ["-fno-honor-nans"], "cs_paged_attn.hip": ["-fno-honor-nans"],
               "cs_paged_fp4_attn.hip": ["-fno-honor-nans"]}


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, src.replace(".hip", ".o"))
    cmd = [HIPCC, *FLAGS, *EXTRA_FLAGS.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{err}")
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def build_lib(jobs: int = 6) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with ThreadPoolExecutor(max_workers=jobs) as ex:
        objs = list(ex.map(_compile, SOURCES))
    r = subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    return LIB


if __name__ == "__main__":
    print(build_lib())
