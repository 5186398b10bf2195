"""Compile the HIP library libpam_lattice.so for gfx950 (in-tree).

Run as ``python -m paper_1907_00641_amd.build``; ``__graft_entry__.build()``
calls :func:`build_library` too.  hipcc cross-compiles without a GPU.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libpam_lattice.so")
SOURCES = ["pam_build.hip", "pam_filter.hip", "pam_block.hip", "pam_probe.hip", "pam_abi.cpp",
           "pam_attn_f32.hip", "pam_attn_f16.hip", "pam_attn_bf16.hip", "pam_attn.cpp",
           "pam_rotary.hip", "pam_norm.hip", "pam_attn_abi.cpp",
           "pam_paged_f32.hip", "pam_paged_f16.hip", "pam_paged_bf16.hip", "pam_paged.cpp",
           "pam_packed_f32.hip", "pam_packed_f16.hip", "pam_packed_bf16.hip", "pam_packed.cpp", "pam_head_norm.hip", "pam_cache.hip", "pam_packed_abi.cpp"]
ARCH = "gfx950"


def hipcc() -> str:
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found (ROCm toolchain required to build the library)")
    return exe


def compile_flags():
    return [
        f"--offload-arch={ARCH}",
        "-O3",
        "-std=c++17",
        "-fPIC",
        "-Wall",
        "-Wno-unused-function",
        # no packed fp32 instructions anywhere in the device code
        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    ]


def build_library(verbose: bool = False) -> str:
    """Compile every source and link the shared library; returns its path."""
    exe = hipcc()
    objdir = os.path.join(PKG, "_build")
    os.makedirs(objdir, exist_ok=True)
    objs, procs = [], []
    for src in SOURCES:  # translation units compile in parallel
        path = os.path.join(CSRC, src)
        obj = os.path.join(objdir, os.path.splitext(src)[0] + ".o")
        lang = ["-x", "hip"] if src.endswith(".hip") else []
        cmd = [exe, *compile_flags(), *lang, "-c", path, "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd)))
        objs.append(obj)
    failed = [src for src, p in procs if p.wait() != 0]
    if failed:
        raise RuntimeError(f"hipcc failed on {failed}")
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [exe, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose="-v" in sys.argv))
