"""Builds libklay.so (HIP kernels + host layerizer + C ABI) for gfx950 with hipcc, in-tree."""
from __future__ import annotations

import os
import shutil
import subprocess
import tempfile

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB_DIR = os.path.join(_HERE, "lib")
LIB_PATH = os.path.join(LIB_DIR, "libklay.so")
SOURCES = ["klay_lib.hip", "klay_head.hip", "klay_head_f32.hip", "klay_head_bf16.hip", "klay_head_f16.hip", "layerize.cpp"]


def hipcc() -> str:
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found; the GPU library cannot be built")
    return exe


def build(verbose: bool = False) -> str:
    """Compile unconditionally and return the library path."""
    os.makedirs(LIB_DIR, exist_ok=True)
    tmp = LIB_PATH + ".tmp.%d" % os.getpid()
    flags = [hipcc(), "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-Wall", "-Wno-unused-command-line-argument"]
    with tempfile.TemporaryDirectory(dir=LIB_DIR) as objects:
        compiles = [flags + ["-c", "-o", os.path.join(objects, f + ".o"), os.path.join(CSRC, f)] for f in SOURCES]
        link = [flags[0], "--offload-arch=gfx950", "-shared", "-o", tmp] + [c[c.index("-o") + 1] for c in compiles]
        if verbose:
            print("\n".join(" ".join(c) for c in compiles + [link]))
        running = [subprocess.Popen(c) for c in compiles]
        failed = [c for c, p in zip(compiles, running) if p.wait() != 0]
        if failed:
            raise subprocess.CalledProcessError(1, failed[0])
        subprocess.check_call(link)
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
