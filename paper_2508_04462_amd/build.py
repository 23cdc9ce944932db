"""Compiles libcard.so (HIP kernels + C ABI) for gfx950, in-tree."""
from __future__ import annotations

import os
import subprocess

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
LIB_PATH = os.path.join(PKG_DIR, "libcard.so")
SOURCES = [
    os.path.join(PKG_DIR, "csrc", "card_api.hip"),
    os.path.join(PKG_DIR, "csrc", "card_serving.hip"),
    os.path.join(PKG_DIR, "csrc", "card_sequences.hip"),
    os.path.join(PKG_DIR, "csrc", "card_cache.cpp"),
]


def build_library(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cmd = [
        hipcc,
        "--offload-arch=gfx950",
        "-O3",
        "-std=c++17",
        "-shared",
        "-fPIC",
        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
        "-I", os.path.join(ROOT, "include"),
        "-I", os.path.join(PKG_DIR, "csrc"),
        "-o", LIB_PATH,
    ] + os.environ.get("CARD_EXTRA_FLAGS", "").split() + SOURCES
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed ({res.returncode}):\n{err}")
    if verbose and err.strip():
        print(err, flush=True)
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(verbose=True))
