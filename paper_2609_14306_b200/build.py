"""Builds the C-ABI CUDA library in-tree with nvcc for sm_100a (no JIT cache, no torch extension)."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
REPO_DIR = os.path.dirname(PKG_DIR)
SOURCES = [os.path.join(PKG_DIR, "csrc", "vp_ce.cu"), os.path.join(PKG_DIR, "csrc", "stream_adamw.cu"),
           os.path.join(PKG_DIR, "csrc", "layer_norm.cu"), os.path.join(PKG_DIR, "csrc", "sequence_loss.cu"),
           os.path.join(PKG_DIR, "csrc", "muon.cu")]
HEADERS = [os.path.join(REPO_DIR, "include", "vp_ce.h"), os.path.join(REPO_DIR, "include", "stream_adamw.h"),
           os.path.join(PKG_DIR, "csrc", "sm100_ptx.cuh"), os.path.join(PKG_DIR, "csrc", "vp_ce_kernels.cuh"),
           os.path.join(REPO_DIR, "include", "vp_ce_types.h"), os.path.join(REPO_DIR, "include", "layer_norm.h"),
           os.path.join(REPO_DIR, "include", "sequence_loss.h"), os.path.join(REPO_DIR, "include", "muon.h"),
           os.path.join(PKG_DIR, "csrc", "muon_kernels.cuh"), os.path.join(PKG_DIR, "csrc", "vp_ce_f32.inc"), os.path.join(PKG_DIR, "csrc", "vp_ce_fixup.cuh")]
LIB_PATH = os.path.join(PKG_DIR, "libvpce.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "--shared", "-Xcompiler", "-fPIC", "-Xptxas", "-v",
]


def find_nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found; cannot build libvpce.so")


def is_stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    return any(os.path.getmtime(p) > t for p in SOURCES + HEADERS)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile csrc/*.cu into libvpce.so next to this file; returns the library path."""
    if not force and not is_stale():
        return LIB_PATH
    cmd = [find_nvcc(), *NVCC_FLAGS, "-I", os.path.join(REPO_DIR, "include"), "-o", LIB_PATH, *SOURCES]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    if verbose:
        sys.stderr.write(res.stdout + res.stderr)
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose=True))
