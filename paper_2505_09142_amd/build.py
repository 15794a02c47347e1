"""Build libelis.so (gfx950) in-tree with hipcc.

    python -m paper_2505_09142_amd.build          # compile every csrc/*.hip, link
Objects go to paper_2505_09142_amd/_build/; the library to
paper_2505_09142_amd/libelis.so. Every call recompiles.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libelis.so")
INCLUDE = os.path.join(ROOT, "include")

ARCH = "gfx950"
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

CFLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
    # keep the compiler from forming packed-fp32 (v_pk_*_f32) instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", INCLUDE, "-I", CSRC,
]


# Per-source extra flags. attention.hip rescales its MFMA accumulators with VALU every key
# tile; keeping them in VGPRs (not AGPRs) avoids a register-file round trip per rescale. Its
# arithmetic never forms a NaN from finite inputs (masked scores are -inf, the running maximum
# starts at -inf and is finite after the first tile), so maxima need no NaN canonicalisation.
# Its kernel arguments, and the product kernels', are preloaded into SGPRs at wave launch (the
# attention work-group's first scalar load is then its work-list entry: 52.5 -> 51.9 us per
# BERT-base layer; the products gain ~0.5 us per launch).
# kv_attention.hip keeps its accumulators in VGPRs for the same reason; its cache may hold NaN, so it honours them.
EXTRA = {
    "attention.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form", "-fno-honor-nans", "-mllvm", "-amdgpu-kernarg-preload-count=16"],
    "kv_attention.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
    "gemm.hip": ["-mllvm", "-amdgpu-kernarg-preload-count=16"],
}


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.basename(src).replace(".hip", ".o"))
    cmd = [HIPCC, *CFLAGS, *EXTRA.get(os.path.basename(src), []), "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj


def build(verbose: bool = True) -> str:
    os.makedirs(BUILD, exist_ok=True)
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.hip")))
    if not srcs:
        raise RuntimeError("no HIP sources found")
    jobs = min(len(srcs), int(os.environ.get("MAX_JOBS", "8")))
    with cf.ThreadPoolExecutor(jobs) as ex:
        objs = list(ex.map(_compile, srcs))
    vscript = os.path.join(BUILD, "exports.map")
    with open(vscript, "w") as f:
        f.write("{ global: elis_*; local: *; };\n")
    tmp = LIB + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs,
           f"-Wl,--version-script={vscript}", "-Wl,--no-undefined"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB} from {len(srcs)} sources", flush=True)
    return LIB


if __name__ == "__main__":
    if shutil.which(HIPCC) is None and not os.path.exists(HIPCC):
        sys.exit(f"hipcc not found at {HIPCC}")
    build()
