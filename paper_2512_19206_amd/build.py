"""Builds libmixkvq.so (HIP, gfx950) in-tree with hipcc."""
from __future__ import annotations

import os
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmixkvq.so")
SOURCES = ["api.hip", "select_kernels.hip", "quantize_kernels.hip", "decode_kernels.hip", "decode_mfma.hip", "decode_mfma_any_lengths.hip",
           "chunk_api.hip", "chunk_kernels.hip", "chunk_few_1.hip", "chunk_few_2.hip", "chunk_few_3.hip", "verify_kernels.hip",
           "decode_mfma_generic_plain.hip", "decode_mfma_generic_g32.hip", "decode_mfma_generic_rh.hip"]
# These kernels never meet a NaN in a maximum: where one is thinkable, every result of a matrix instruction is copied ("quieted")
# before it is compared.
EXTRA_FLAGS = {src: ["-fno-honor-nans"] for src in ("chunk_kernels.hip", "chunk_few_1.hip", "chunk_few_2.hip", "chunk_few_3.hip")}
OBJ_DIR = os.path.join(HERE, "_build")      # object files (git-ignored)


def hipcc_path() -> str:
    for cand in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def _flags():
    return ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-Wall", "-Wno-unused-function", "-fno-strict-aliasing",
            "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(OBJ_DIR, os.path.splitext(src)[0] + ".o")
    cmd = [hipcc_path()] + _flags() + EXTRA_FLAGS.get(src, []) + ["-c", os.path.join(CSRC, src), "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n" + res.stdout + res.stderr)
    if verbose and res.stderr:
        print(res.stderr)
    return obj


def build_library(verbose: bool = False) -> str:
    """Compile every HIP source for gfx950 (the translation units in parallel) and link the shared library."""
    from concurrent.futures import ThreadPoolExecutor
    os.makedirs(OBJ_DIR, exist_ok=True)
    jobs = min(len(SOURCES), max(1, min(os.cpu_count() or 1, int(os.environ.get("MAX_JOBS", "8")))))
    with ThreadPoolExecutor(max_workers=jobs) as pool:
        objs = list(pool.map(lambda src: _compile(src, verbose), SOURCES))
    cmd = [hipcc_path(), "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objs
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("link failed:\n" + res.stdout + res.stderr)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
