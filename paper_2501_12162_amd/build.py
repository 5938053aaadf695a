"""Builds ``libadaserve.so`` (the C ABI in include/adaserve.h) for gfx950.

Usage: ``python -m paper_2501_12162_amd.build`` or ``build()`` from Python.
The library is written in-tree to ``paper_2501_12162_amd/_build/``.
"""
from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(PKG, "_build")
LIB_PATH = os.path.join(BUILD_DIR, "libadaserve.so")
ARCH = "gfx950"


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.cpp")))


# Beside the flags of every source: prompt attention holds its matrix
# products' results in vector registers (the accumulation registers, which the
# vector ALUs cannot read, would take a move per score).
FILE_FLAGS = {"prompt_attn.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=true"]}


def build(verbose: bool = False) -> str:
    """Compile every HIP/C++ source of the library into one shared object."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    with tempfile.TemporaryDirectory(dir=BUILD_DIR) as work:
        flags = ["--offload-arch=" + ARCH, "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
                 # keep the compiler from forming packed fp32 VALU ops
                 "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-I", INCLUDE, "-I", CSRC]

        def run(cmd):
            proc = subprocess.run(cmd, capture_output=True, text=True)
            if proc.returncode != 0:
                sys.stderr.write(proc.stdout + proc.stderr)
                raise RuntimeError("building libadaserve.so failed")
            if verbose:
                noise = "is not a recognized feature for this target"
                sys.stderr.write("".join(l + "\n" for l in (proc.stdout + proc.stderr).splitlines() if noise not in l))

        def compile_one(src):
            name = os.path.basename(src)
            obj = os.path.join(work, name + ".o")
            run([hipcc(), *flags, *FILE_FLAGS.get(name, []), "-c", src, "-o", obj])
            return obj

        with ThreadPoolExecutor(max_workers=8) as pool:
            objs = list(pool.map(compile_one, sources()))
        tmp = os.path.join(work, "libadaserve.so")
        run([hipcc(), "--offload-arch=" + ARCH, "-shared", "-fPIC", *objs, "-o", tmp])
        os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
