"""Build ``libdigest.so`` in-tree for gfx950.

Host code (``HOST_SOURCES``) is plain C++ built with g++ against the HIP
runtime headers; the kernels (``KERNEL_SOURCES``) are built with hipcc for
gfx950.  Packed-fp32 instructions are disabled for all GPU code.

    python -m paper_2206_00057_amd.build
"""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libdigest.so")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
ARCH = "gfx950"
HOST_SOURCES = ("digest_host", "digest_train")
KERNEL_SOURCES = ("digest_kernels", "norm_kernels", "orth_kernels")

HIPCC_FLAGS = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-Wall", "-I", INCLUDE, "-I", CSRC]
CXX_FLAGS = ["-O2", "-std=c++17", "-fPIC", "-Wall", "-Wextra", "-Wno-unused-parameter",
             "-D__HIP_PLATFORM_AMD__", "-I", INCLUDE, "-I", CSRC, "-I", os.path.join(ROCM, "include")]


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in res.stdout.splitlines()
                    if "packed-fp32-ops" not in l and "not a recognized feature" not in l)
    if res.returncode != 0:
        raise RuntimeError(f"build step failed ({res.returncode}): {' '.join(cmd)}\n{out}")
    if verbose and out.strip():
        print(out)


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    jobs, objs = [], []
    for name in HOST_SOURCES:
        objs.append(os.path.join(BUILD, name + ".o"))
        jobs.append(["g++", *CXX_FLAGS, "-c", os.path.join(CSRC, name + ".cpp"), "-o", objs[-1]])
    for name in KERNEL_SOURCES:
        objs.append(os.path.join(BUILD, name + ".o"))
        jobs.append([os.path.join(ROCM, "bin", "hipcc"), *HIPCC_FLAGS, "-c",
                     os.path.join(CSRC, name + ".hip"), "-o", objs[-1]])
    with concurrent.futures.ThreadPoolExecutor(len(jobs)) as pool:
        list(pool.map(lambda cmd: _run(cmd, verbose), jobs))
    tmp = LIB + f".tmp{os.getpid()}"
    _run([os.path.join(ROCM, "bin", "hipcc"), f"--offload-arch={ARCH}", "-shared", "-fPIC",
          *objs, "-o", tmp], verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
