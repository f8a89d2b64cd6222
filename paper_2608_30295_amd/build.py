"""Build the CateKV HIP library for gfx950 in-tree (``libcatekv.so``).

Usage: ``python -m paper_2608_30295_amd.build`` (or ``build()`` from Python).
hipcc cross-compiles for gfx950, so this runs without a GPU.
"""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libcatekv.so")
ARCH = "gfx950"
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")

HIP_SOURCES = ["decode.hip", "prefill.hip", "retrieve.hip", "score_rowstats.hip", "score_colmass.hip", "score_obs.hip", "score_obsb.hip", "cv.hip",
               "q8.hip", "attend_dense.hip", "attend_i8.hip", "attend_e4m3.hip", "evict.hip",
               "paged_pages.hip", "paged_tile.hip", "paged_tile_f32.hip", "paged_stream.hip", "paged_join.hip"]
HOST_SOURCES = ["api.cpp", "cache_api.cpp", "paged_api.cpp"]

# Packed fp32 ops are kept out of the device code: hipcc only emits them when
# asked, and the build never asks.
DEVICE_FLAGS = ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
COMMON = ["-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function", f"-I{INCLUDE}"]


def _hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found: the ROCm toolchain is required to build libcatekv.so")


def _cxx() -> str:
    return shutil.which("g++") or shutil.which("c++") or "g++"


def _run(cmd):
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in r.stdout.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"command failed ({r.returncode}): {' '.join(cmd)}\n{out}")
    return out


def build(verbose: bool = False) -> str:
    """Compile every source and link libcatekv.so; returns its path."""
    hipcc = _hipcc()
    bdir = os.path.join(HERE, "_build")
    os.makedirs(bdir, exist_ok=True)
    objs = []
    cmds = []
    for src in HIP_SOURCES:
        obj = os.path.join(bdir, src + ".o")
        cmds.append([hipcc, "-x", "hip", f"--offload-arch={ARCH}", *COMMON, *DEVICE_FLAGS, "-c",
                     os.path.join(CSRC, src), "-o", obj])
        objs.append(obj)
    for src in HOST_SOURCES:
        # plain host C++ against the HIP runtime API
        obj = os.path.join(bdir, src + ".o")
        cmds.append([_cxx(), *COMMON, "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", "-c",
                     os.path.join(CSRC, src), "-o", obj])
        objs.append(obj)
    with concurrent.futures.ThreadPoolExecutor(max_workers=len(cmds)) as ex:
        for out in ex.map(_run, cmds):
            if verbose and out.strip():
                print(out)
    tmp = LIB + ".tmp"
    _run([hipcc, f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp,
          f"-L{ROCM}/lib", "-lamdhip64", f"-Wl,-rpath,{ROCM}/lib"])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
