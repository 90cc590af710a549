"""Builds the CUDA library in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libtgrad.so")
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"]


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    deps.append(os.path.join(os.path.dirname(HERE), "include", "tgrad.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile libtgrad.so if it is missing or older than its sources."""
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "nvcc")

    def run(args):
        res = subprocess.run([nvcc] + args, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
        return res.stderr

    with tempfile.TemporaryDirectory() as tmp:      # the sources side by side, then the library
        objects = [os.path.join(tmp, os.path.basename(f) + ".o") for f in sources()]
        compile_flags = NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else [])
        with ThreadPoolExecutor(len(objects)) as pool:
            logs = list(pool.map(lambda fo: run(compile_flags + ["-c", "-o", fo[1], fo[0]]), zip(sources(), objects)))
        run(NVCC_FLAGS + ["-shared", "-o", LIB] + objects)
    if verbose:
        print("".join(logs))
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
