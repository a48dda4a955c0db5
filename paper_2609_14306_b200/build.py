"""Builds the C-ABI CUDA library in-tree with nvcc for sm_100a (no JIT cache, no torch extension)."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
REPO_DIR = os.path.dirname(PKG_DIR)
SOURCES = [os.path.join(PKG_DIR, "csrc", "vp_ce.cu"), os.path.join(PKG_DIR, "csrc", "stream_adamw.cu"),
           os.path.join(PKG_DIR, "csrc", "layer_norm.cu"), os.path.join(PKG_DIR, "csrc", "sequence_loss.cu"),
           os.path.join(PKG_DIR, "csrc", "muon.cu"), os.path.join(PKG_DIR, "csrc", "rms_norm.cu"),
           os.path.join(PKG_DIR, "csrc", "token_logp.cu"), os.path.join(PKG_DIR, "csrc", "fp8_blocks.cu")]
HEADERS = [os.path.join(REPO_DIR, "include", "vp_ce.h"), os.path.join(REPO_DIR, "include", "stream_adamw.h"),
           os.path.join(PKG_DIR, "csrc", "sm100_ptx.cuh"), os.path.join(PKG_DIR, "csrc", "vp_ce_kernels.cuh"),
           os.path.join(REPO_DIR, "include", "vp_ce_types.h"), os.path.join(REPO_DIR, "include", "layer_norm.h"),
           os.path.join(REPO_DIR, "include", "sequence_loss.h"), os.path.join(REPO_DIR, "include", "muon.h"),
           os.path.join(REPO_DIR, "include", "rms_norm.h"), os.path.join(PKG_DIR, "csrc", "row_kernels.cuh"),
           os.path.join(REPO_DIR, "include", "token_logp.h"), os.path.join(REPO_DIR, "include", "fp8_blocks.h"),
           os.path.join(PKG_DIR, "csrc", "token_logp_kernels.cuh"),
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
    nvcc = find_nvcc()

    def run(*args: str) -> str:
        res = subprocess.run([nvcc, *args], capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
        return res.stdout + res.stderr

    # one process per source: the longest decides
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, os.path.basename(src) + ".o") for src in SOURCES]
        flags = [f for f in NVCC_FLAGS if f != "--shared"]
        compile_one = lambda src, obj: run(*flags, "-c", "-I", os.path.join(REPO_DIR, "include"), "-o", obj, src)  # noqa: E731
        with ThreadPoolExecutor(max_workers=min(len(SOURCES), os.cpu_count() or 1)) as pool:
            log = "".join(pool.map(compile_one, SOURCES, objects))
        log += run(*NVCC_FLAGS, "-o", LIB_PATH, *objects)
    if verbose:
        sys.stderr.write(log)
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose=True))
