"""Builds libngsgd.so (HIP, gfx950) in-tree with hipcc."""
from __future__ import annotations

import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB_PATH = os.path.join(HERE, "libngsgd.so")
SOURCES = [os.path.join(HERE, "csrc", name) for name in ("ngsgd.hip", "layer_norm.hip", "adamw.hip")]

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
    # no packed fp32 instructions: some of their forms have given wrong results on this hardware
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-result",
]


def find_hipcc() -> str:
    for cand in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found: the ngsgd library needs the ROCm toolchain to build")


def build(verbose: bool = False) -> str:
    """Compiles every source (side by side) and links them; raises with the compiler's output if one fails."""
    hipcc = find_hipcc()
    objects = os.path.join(HERE, "_build")
    os.makedirs(objects, exist_ok=True)
    include = ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "csrc")]

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        return subprocess.run(cmd, capture_output=True, text=True)

    def compile_one(source):
        return run([hipcc, *HIPCC_FLAGS, *include, "-c", "-o", os.path.join(objects, os.path.basename(source) + ".o"), source])

    with ThreadPoolExecutor(max_workers=min(len(SOURCES), os.cpu_count() or 1)) as pool:
        results = list(pool.map(compile_one, SOURCES))
    if all(r.returncode == 0 for r in results):
        results.append(run([hipcc, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", LIB_PATH,
                            *(os.path.join(objects, os.path.basename(s) + ".o") for s in SOURCES)]))
    for proc in results:
        if proc.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + proc.stdout + proc.stderr)
        if verbose and proc.stderr.strip():
            print(proc.stderr)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
