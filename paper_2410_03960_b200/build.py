"""Builds the CUDA library in-tree:  python -m paper_2410_03960_b200.build [--force] [--library]

One nvcc invocation compiles every .cu under csrc/ for sm_100a into libswiftkv.so next to this file; then g++ compiles
csrc/verify_py.cpp, a Python extension against torch's headers, into _verify.so.  --library builds the C library alone, which needs
neither torch nor Python's headers.  nvcc cross-compiles without a GPU, so this also runs on a CPU-only machine.
"""
from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libswiftkv.so")
EXT = os.path.join(HERE, "_verify.so")      # tensor marshalling of the verification-step operators (no kernels)
SOURCES = ["api.cu", "elementwise.cu", "gemm_simt.cu", "gemm_tc.cu", "attention_simple.cu", "attention_tc.cu", "tail.cu", "tail_noalloc.cu", "kv_fp8.cu", "simscore.cu", "distill.cu",
           "page_plan.cu", "qk_rope.cu", "tree_attention.cu", "logprobs.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "--use_fast_math",
              "-Xcompiler", "-fPIC", "-shared", "-Xptxas", "-v"]


def _nvcc() -> str:
    return os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")


def _torch_version_file() -> str:
    spec = importlib.util.find_spec("torch")
    return os.path.join(os.path.dirname(spec.origin), "version.py") if spec and spec.origin else ""


def _ext_stale() -> bool:
    """Older than its sources or than the torch that it would be loaded into (one of another version refuses to load, see verify.py)."""
    if not os.path.exists(EXT):
        return True
    t = os.path.getmtime(EXT)
    deps = (os.path.join(CSRC, "verify_py.cpp"), os.path.join(HERE, "..", "include", "swiftkv.h"), _torch_version_file())
    return any(os.path.exists(d) and os.path.getmtime(d) > t for d in deps)


def build_ext(verbose: bool = False) -> str:
    """csrc/verify_py.cpp -> _verify.so."""
    import sysconfig

    import torch
    torch_dir = os.path.dirname(torch.__file__)
    nvcc = os.path.realpath(shutil.which(_nvcc()) or _nvcc())
    inc = [os.path.join(torch_dir, "include"), os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"),
           os.path.join(os.path.dirname(os.path.dirname(nvcc)), "include"), sysconfig.get_paths()["include"]]
    libs = os.path.join(torch_dir, "lib")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           f'-DSWIFTKV_TORCH="{torch.__version__}"'] + [f"-I{i}" for i in inc] + \
        [os.path.join(CSRC, "verify_py.cpp"), "-o", EXT, f"-L{libs}", "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or proc.returncode != 0:
        sys.stderr.write(proc.stdout + proc.stderr)
    if proc.returncode != 0:
        raise RuntimeError("g++ failed building _verify.so")
    return EXT


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if not f.endswith(".cpp")] + [os.path.join(HERE, "..", "include", "swiftkv.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """The library, then the extension: what fails of the second leaves the first built."""
    build_library(force, verbose)
    if force or _ext_stale():
        build_ext(verbose)
    return LIB


def build_library(force: bool = False, verbose: bool = False) -> str:
    """csrc/*.cu -> libswiftkv.so."""
    if not force and not _stale():
        return LIB
    cmd = [_nvcc()] + NVCC_FLAGS + [os.path.join(CSRC, s) for s in SOURCES] + ["-o", LIB]
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or proc.returncode != 0:
        sys.stderr.write(proc.stdout + proc.stderr)
    if proc.returncode != 0:
        raise RuntimeError("nvcc failed building libswiftkv.so")
    # register / spill / shared-memory report of ptxas: scratch output, kept out of the source tree
    log_dir = os.environ.get("SWIFTKV_BUILD_LOG_DIR", os.path.join(HERE, "..", "gpurun_out"))
    try:
        os.makedirs(log_dir, exist_ok=True)
        with open(os.path.join(log_dir, "build_ptxas.log"), "w") as f:
            f.write(proc.stdout + proc.stderr)
    except OSError:
        pass
    return LIB


if __name__ == "__main__":
    print((build_library if "--library" in sys.argv else build)(force="--force" in sys.argv, verbose=True))
