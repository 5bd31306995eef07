"""Compile the HIP sources of libbmgd for gfx950, and the module that reads torch tensors, into this package directory."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libbmgd.so")
SOURCES = ["bmgd_api.hip", "perm_kernel.hip", "glm_kernels.hip", "glm_split_kernel.hip", "glm_narrow_kernel.hip", "softmax_kernels.hip", "softmax_chain_kernel.hip", "softmax_pass_kernel.hip", "gram_kernels.hip", "gram_fused_kernel.hip", "gram_products.hip", "reader.hip", "noalloc.hip", "gated_block.hip", "gated_bf16.hip", "gated_f16.hip", "adamw_kernel.hip"]
TENSORS = os.path.join(HERE, "_tensors.so")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wall", "-Wno-unused-function"]


def hipcc() -> str:
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found")
    return exe


def tensors_command() -> list[str]:
    """Of csrc/tensors.cpp: a Python module on torch's C++ headers, host code only."""
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    lib = os.path.join(root, "lib")
    return [shutil.which("g++") or "c++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            f"-isystem{os.path.join(root, 'include')}", f"-isystem{os.path.join(root, 'include', 'torch', 'csrc', 'api', 'include')}", f"-isystem{sysconfig.get_paths()['include']}",
            os.path.join(CSRC, "tensors.cpp"), "-o", TENSORS, f"-L{lib}", "-ltorch_python", "-ltorch_cpu", "-lc10", f"-Wl,-rpath,{lib}"]


def build(verbose: bool = True) -> str:
    """Always recompiles; returns the path of the shared library."""
    cc = hipcc()
    noise = "is not a recognized feature for this target"

    def compile_one(src: str) -> str:
        obj = os.path.join(CSRC, src.replace(".hip", ".o"))
        cmd = [cc, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        res = subprocess.run(cmd, capture_output=True, text=True)
        err = "\n".join(ln for ln in res.stderr.splitlines() if noise not in ln)
        if res.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{err}")
        if verbose and err.strip():
            print(err, file=sys.stderr)
        return obj

    def compile_tensors() -> None:
        cmd = tensors_command()
        if verbose:
            print(" ".join(cmd), flush=True)
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError(f"tensors.cpp failed:\n{res.stderr}")

    # the sources are independent: compile them side by side (a handful of processes)
    from concurrent.futures import ThreadPoolExecutor
    with ThreadPoolExecutor(max_workers=min(len(SOURCES), 8)) as pool:
        tensors = pool.submit(compile_tensors)
        objs = list(pool.map(compile_one, SOURCES))
        tensors.result()
    cmd = [cc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{res.stderr}")
    return LIB


if __name__ == "__main__":
    print(build())
