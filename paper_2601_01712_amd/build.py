"""Builds librelaygr.so (the C-ABI library) in-tree with hipcc for gfx950."""
from __future__ import annotations

import os
import shutil
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "librelaygr.so")
SOURCES = ["engine.hip", "cache_ops.hip", "rotary.hip", "scored_ops.hip", "evict.hip", "kv_pool.cpp", "expander.hip", "admission.cpp"]
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]


def hipcc_path() -> str:
    for cand in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def _run(cmd, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    # the host pass warns that it does not know the packed-fp32 target feature; that is expected
    noise = "is not a recognized feature for this target"
    err = "\n".join(ln for ln in res.stderr.splitlines() if noise not in ln)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + err)
    if verbose and err.strip():
        print(err)


def build(verbose: bool = False) -> str:
    """Compiles every source of the library, all of them at once (the longest, the attention kernels', is half of the work), and links them; raises on
    failure; returns the library path."""
    hipcc, compile_flags = hipcc_path(), [f for f in FLAGS if f != "-shared"]
    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(len(SOURCES)) as pool:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        # (list(): a failure is raised here)
        list(pool.map(lambda s, o: _run([hipcc, *compile_flags, "-x", "hip", "-c", os.path.join(CSRC, s), "-o", o], verbose), SOURCES, objects))
        _run([hipcc, *FLAGS, *objects, "-o", LIB], verbose)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
