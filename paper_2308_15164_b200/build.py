"""Builds the C-ABI library (sm_100a only) from csrc/*.cu into paper_2308_15164_b200/libabs_sgd.so, and the extension
module of llm.py (host code: its functions on PyTorch tensors) from csrc/llm_torch.cpp into paper_2308_15164_b200/_llm.so.
Without PyTorch the library alone is built: its C interface does not need it.
"""

from __future__ import annotations

import glob
import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libabs_sgd.so")
MODULE_SOURCE = os.path.join(CSRC, "llm_torch.cpp")
MODULE = os.path.join(HERE, "_llm.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-shared", "-Xcompiler", "-fPIC", "--threads", "4", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _older(target, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def needs_build() -> bool:
    return _older(LIB, sources() + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(
        os.path.join(ROOT, "include", "*.h")) + [os.path.abspath(__file__)])


def _run(cmd, verbose=False):
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if verbose or res.returncode != 0:
        print(res.stdout)
    if res.returncode != 0:
        raise RuntimeError(cmd[0] + " failed: " + " ".join(cmd))


def _module_command(target):
    import torch

    at = os.path.dirname(torch.__file__)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    include = [os.path.join(ROOT, "include"), os.path.join(at, "include"), os.path.join(at, "include", "torch", "csrc", "api", "include"),
               os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"] + ["-I" + d for d in include] + [
        MODULE_SOURCE, "-o", target, "-L" + os.path.join(at, "lib"), "-ltorch_python", "-ltorch_cuda", "-ltorch_cpu", "-lc10_cuda", "-lc10",
        "-L" + HERE, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN"]


def build(force: bool = False, verbose: bool = False, extra=()) -> str:
    if force or needs_build():
        _run([os.environ.get("NVCC", "nvcc")] + NVCC_FLAGS + list(extra) + (["-Xptxas", "-v"] if verbose else []) + ["-o", LIB] + sources(), verbose)
    if importlib.util.find_spec("torch") is None:
        return LIB
    if force or _older(MODULE, [MODULE_SOURCE, os.path.join(ROOT, "include", "abs_llm.h"), os.path.join(ROOT, "include", "abs_sgd.h"),
                                os.path.abspath(__file__)]):
        _run(_module_command(MODULE), verbose)
    return LIB


if __name__ == "__main__":
    build(force="--force" in sys.argv, verbose="-v" in sys.argv)
    print(LIB)
