"""Builds libadloco.so in-tree with nvcc for sm_100a, and beside it the extension module that marshals torch tensors
for the calls that run once a layer (_tensor_calls.so, host code only).

    python -m paper_2508_18182_b200.build [--force] [--verbose]
"""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libadloco.so")
CALLS = os.path.join(PKG, "_tensor_calls.so")
SOURCES = ["api.cu", "stream_kernels.cu", "gram_kernels.cu", "block_api.cu", "block_kernels.cu",
           "blockscale_gemm.cu"]
HEADERS = ["common.cuh", os.path.join("..", "..", "include", "adloco.h")]


def _older(target, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps if os.path.exists(d))


def _stale() -> bool:
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS] + [os.path.abspath(__file__)]
    deps += [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    return _older(LIB, deps)


def _build_calls(force: bool, verbose: bool) -> None:
    import sysconfig
    try:
        import torch
    except ImportError:
        torch = None
    if torch is None or torch.version.cuda is None:
        # the library needs nvcc alone, and all but the operators between the linear layers is reached without the module
        sys.stderr.write("_tensor_calls.so is not built: it needs torch with CUDA\n")
        return
    source = os.path.join(CSRC, "tensor_calls.cpp")
    # it is good for one torch and one Python: which ones it was compiled against stands beside it
    stamp = os.path.splitext(CALLS)[0] + ".stamp"
    against = f"torch {torch.__version__}, Python {sys.version_info.major}.{sys.version_info.minor}\n"
    if not force and not _older(CALLS, [source, os.path.join(CSRC, HEADERS[-1]), os.path.abspath(__file__)]):
        if os.path.exists(stamp) and open(stamp).read() == against:
            return
    root = os.path.dirname(torch.__file__)
    includes = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
                sysconfig.get_paths()["include"], os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")]
    cmd = [os.environ.get("CXX", "g++"), "-shared", "-o", CALLS, "-std=c++17", "-O2", "-Wall", "-fPIC", "-fvisibility=hidden", source]
    cmd += ["-I" + d for d in includes]
    cmd += ["-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda",
            "-L" + PKG, "-l:libadloco.so", "-Wl,-rpath,$ORIGIN"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
    if res.returncode != 0:
        raise RuntimeError("building _tensor_calls.so failed")
    with open(stamp, "w") as f:
        f.write(against)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles every .cu of the library into paper_2508_18182_b200/libadloco.so, and the marshalling module where torch
    has CUDA."""
    if not force and not _stale():
        _build_calls(force, verbose)
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-shared", "-o", LIB, "-std=c++17", "-O3", "-lineinfo",
           "-gencode", "arch=compute_100a,code=sm_100a",
           "-Xcompiler", "-fPIC,-O3,-Wall,-fvisibility=hidden",
           "-Xptxas", "-v" if verbose else "-warn-spills",
           "-DADLOCO_BUILD", "--threads", "0"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed building libadloco.so")
    _build_calls(force, verbose)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
