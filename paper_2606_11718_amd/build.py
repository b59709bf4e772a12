"""Build libccl.so (host plan + HIP kernels for gfx950 + C ABI) in-tree.

    python -m paper_2606_11718_amd.build
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OUT_DIR = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libccl.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
# -packed-fp32-ops: keep the compiler from forming packed fp32 VALU ops.
# Code object v5: loadable by the HIP runtime bundled with torch (ROCm 7.0)
# as well as by the system ROCm 7.2 runtime.
HIP_FLAGS = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}", "-Wall", "-Wno-inline-asm", "-mcode-object-version=5",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-I", os.path.join(ROOT, "include"), "-I", CSRC]
HOST_FLAGS = ["-O3", "-std=c++17", "-fPIC", "-pthread", "-Wall", "-Wextra", "-I", CSRC]

SOURCES = [
    ("host/plan.cpp", "host"),       # plain C++, no HIP
    ("host/l2sim.cpp", "host"),
    ("host/train.cpp", "host"),
    ("ccl_api.cpp", "hip"),
    ("ccl_ops.cpp", "hip"),
    ("ccl_train.cpp", "hip"),
    ("kernels/pack.hip", "hip"),
    ("kernels/gemm.hip", "hip"),
    ("kernels/gemm_fused.hip", "hip"),
    ("kernels/moe.hip", "hip"),
    ("kernels/newton_schulz.hip", "hip"),
    ("kernels/grouped.hip", "hip"),
    ("kernels/cross_entropy.hip", "hip"),
    ("kernels/adamw.hip", "hip"),
]


def _compile(src: str, kind: str) -> str:
    path = os.path.join(CSRC, src)
    obj = os.path.join(OUT_DIR, src.replace("/", "_") + ".o")
    if kind == "host":
        cmd = ["g++"] + HOST_FLAGS + ["-c", path, "-o", obj]
    else:
        cmd = [HIPCC] + HIP_FLAGS + ["-x", "hip", "-c", path, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj


def build(verbose: bool = False) -> str:
    """Compile every source and link libccl.so; returns the library path."""
    os.makedirs(OUT_DIR, exist_ok=True)
    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(lambda s: _compile(*s), SOURCES))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, "-shared", "-fPIC", f"--offload-arch={ARCH}", "-mcode-object-version=5", "-pthread", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}")
    return LIB


def clean() -> None:
    shutil.rmtree(OUT_DIR, ignore_errors=True)
    if os.path.exists(LIB):
        os.remove(LIB)


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
