"""Builds libngsgd.so (HIP, gfx950) in-tree with hipcc alone, and where torch and g++ are there the binding's helper _tensors.so (host code)."""
from __future__ import annotations

import os
import shutil
import subprocess
import sysconfig
import warnings
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB_PATH = os.path.join(HERE, "libngsgd.so")
SOURCES = [os.path.join(HERE, "csrc", name) for name in ("ngsgd.hip", "layer_norm.hip", "adamw.hip", "embedding.hip", "cross_entropy.hip", "grad_norm.hip")]

BINDING_PATH = os.path.join(HERE, "_tensors.so")
BINDING_SOURCE = os.path.join(HERE, "csrc", "tensors.cpp")

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


def binding_command():
    """g++ on the binding's helper, against the Python and the torch that run this; None where there is no torch or no g++."""
    try:
        import torch
        from torch.utils import cpp_extension
    except ImportError:
        return None
    if shutil.which("g++") is None:
        return None
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I", sysconfig.get_paths()["include"]]
    for path in cpp_extension.include_paths():
        cmd += ["-isystem", path]
    cmd += ["-o", BINDING_PATH, BINDING_SOURCE]
    for path in cpp_extension.library_paths():
        cmd += ["-L", path, f"-Wl,-rpath,{path}"]
    return cmd + ["-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10"]


def build(verbose: bool = False) -> str:
    """Compiles every source (side by side) and links them, and compiles the binding's helper; raises with the compiler's output if one fails."""
    hipcc = find_hipcc()
    objects = os.path.join(HERE, "_build")
    os.makedirs(objects, exist_ok=True)
    include = ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "csrc")]
    binding = binding_command()

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        return subprocess.run(cmd, capture_output=True, text=True)

    def compile_one(source):
        return run([hipcc, *HIPCC_FLAGS, *include, "-c", "-o", os.path.join(objects, os.path.basename(source) + ".o"), source])

    with ThreadPoolExecutor(max_workers=min(len(SOURCES) + 1, os.cpu_count() or 1)) as pool:
        helper = pool.submit(run, binding) if binding is not None else None
        results = list(pool.map(compile_one, SOURCES))
        if all(r.returncode == 0 for r in results):
            results.append(run([hipcc, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", LIB_PATH,
                                *(os.path.join(objects, os.path.basename(s) + ".o") for s in SOURCES)]))
    if helper is not None:
        results.append(helper.result())
    for proc in results:
        if proc.returncode != 0:
            raise RuntimeError(f"{os.path.basename(proc.args[0])} failed:\n" + proc.stdout + proc.stderr)
        if verbose and proc.stderr.strip():
            print(proc.stderr)
    if helper is None:
        warnings.warn("no torch or no g++: built without _tensors.so, which GradientNorm needs")
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
