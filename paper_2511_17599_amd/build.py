"""Builds libflce.so (the C-ABI library) for gfx950 with hipcc, in-tree.

    python -m paper_2511_17599_amd.build

hipcc cross-compiles without a GPU.  The packed-fp32 target feature is switched
off for all device code of this library.  Launch arguments come preloaded in scalar
registers (the first 16 words): a kernel's first loads otherwise wait for two of its
argument segment, 0.3 to 0.4 us of a forward of 14 us (334 x 320 x 2142).
"""
from __future__ import annotations

import os
import shutil
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
SRC = os.path.join(PKG, "csrc", "flce.hip")
SOURCES = [SRC] + [os.path.join(PKG, "csrc", f) for f in ("topk.hip", "distill.hip")]
LIB = os.path.join(PKG, "libflce.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-mllvm", "-amdgpu-kernarg-preload-count=16",
    "-Wno-unused-command-line-argument",
]


def hipcc_path():
    return shutil.which("hipcc") or "/opt/rocm/bin/hipcc"


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + res.stdout + res.stderr)


def build_library(verbose=False):
    """Compiles the sources under csrc/ side by side and links them into libflce.so next to this file; returns its path."""
    flags = [f for f in HIPCC_FLAGS if f != "-shared"]
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, os.path.basename(s) + ".o") for s in SOURCES]
        with ThreadPoolExecutor(len(SOURCES)) as pool:
            list(pool.map(lambda so: _run([hipcc_path(), *flags, "-c", so[0], "-o", so[1]], verbose), zip(SOURCES, objects)))
        _run([hipcc_path(), "--offload-arch=gfx950", "-fPIC", "-shared", *objects, "-o", LIB + ".tmp"], verbose)
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
