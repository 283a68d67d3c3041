"""Build libcep.so (HIP kernels + C ABI) for gfx950 in-tree with hipcc.

Usage: python -m paper_2609_33252_amd.build   (or __graft_entry__.build()).
Always recompiles every source; objects go to paper_2609_33252_amd/_build/.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libcep.so")
OBJ = os.path.join(HERE, "_build")
ARCH = "gfx950"

SOURCES = ["route.hip", "gemm.hip", "gemm_bf16.hip", "gemm_fp8.hip", "gemm_mx.hip",
           "gemm_rows.hip", "gemm_rows_bf16.hip", "norm.hip", "gate.hip", "dispatch.hip",
           "dense.hip", "dense_rows.hip", "runtime.hip", "profile.cpp", "oewf.cpp"]
# Per-source extra flags.  The e4m3 GEMMs promote every MFMA result with
# VALU arithmetic; taking MFMA results in VGPRs saves one accvgpr read per
# promoted element.
EXTRA = {"gemm_fp8.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
         "gemm_rows.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"]}

# -packed-fp32-ops: keep the compiler from forming v_pk_{add,mul,fma}_f32.
CFLAGS = ["-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden", f"--offload-arch={ARCH}",
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
          "-Wall", "-Wno-unused-function", "-I", os.path.join(ROOT, "include")]


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found (ROCm toolchain required to build libcep)")


def _run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"command failed ({r.returncode}): {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    # the host pass does not know the packed-fp32 feature; that warning is expected
    noise = [l for l in (r.stderr or "").splitlines() if l.strip() and "packed-fp32-ops" not in l]
    if noise:
        sys.stderr.write("\n".join(noise) + "\n")


def build(verbose: bool = False) -> str:
    cc = hipcc()
    os.makedirs(OBJ, exist_ok=True)
    objs = []
    cmds = []
    for src in SOURCES:
        o = os.path.join(OBJ, os.path.splitext(src)[0] + ".o")
        objs.append(o)
        cmds.append([cc, *CFLAGS, *EXTRA.get(src, []), "-c", os.path.join(CSRC, src), "-o", o])
    with ThreadPoolExecutor(min(len(cmds), os.cpu_count() or 1)) as ex:
        list(ex.map(_run, cmds))
    tmp = OUT + ".tmp"
    _run([cc, "-shared", f"--offload-arch={ARCH}", "-fvisibility=hidden", "-o", tmp, *objs])
    os.replace(tmp, OUT)
    if verbose:
        print("built", OUT)
    return OUT


if __name__ == "__main__":
    build(verbose=True)
