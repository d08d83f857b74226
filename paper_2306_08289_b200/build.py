"""Compile the CUDA library for sm_100a into paper_2306_08289_b200/liba2cid2.so, and, where torch with CUDA is installed, the host side of the operators' usual calls into
_calls.so (in-tree). The library needs nvcc alone. _calls.so is tied to one version of torch, which is noted beside it: another one has it built again.

Extra nvcc flags for experiments may be given in the environment variable A2CID2_NVCC_FLAGS, e.g.
"-DA2_EVENT_THREADS=512" (threads per CTA of the event kernel) or "-DA2_TUNING_KNOBS=1" (a build whose
launch shapes can be overridden from the environment, see csrc/a2cid2_internal.h). The default build has
no such flags and reads no tuning variable at run time."""
from __future__ import annotations

import importlib.metadata
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "liba2cid2.so")
CALLS = os.path.join(HERE, "_calls.so")
CALLS_SOURCE = "torch_calls.cpp"
SOURCES = ["api.cu", "kernels.cu", "scheduler.cpp", "spectral.cpp",
           "lm_api.cu", "embed.cu", "gemm_sm100.cu", "vocab_loss.cu", "vocab_loss_few.cu", "orthogonalize.cu",
           "lm_train_api.cu", "rms_norm.cu", "route.cu", "clip.cu"]


def _nvcc() -> str:
    cand = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found: the CUDA library cannot be built")
    return cand


def _older(built: str, sources) -> bool:
    return not os.path.exists(built) or any(os.path.getmtime(p) > os.path.getmtime(built) for p in sources)


def _stale() -> bool:
    """Whether the library has to be built."""
    return _older(LIB, [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != CALLS_SOURCE] + [os.path.join(INCLUDE, "a2cid2.h")])


def torch_version():
    """That of the torch that is installed, found without importing it; None without one, or without its CUDA libraries."""
    try:
        spec = importlib.util.find_spec("torch")
        version = importlib.metadata.version("torch")
    except (ImportError, ValueError):  # PackageNotFoundError is an ImportError
        return None
    places = list(spec.submodule_search_locations or []) if spec else []
    return version if any(os.path.exists(os.path.join(p, "lib", "libc10_cuda.so")) for p in places) else None


def calls_version():
    """The version of torch that _calls.so has been built for, or None."""
    try:
        with open(CALLS + ".torch") as f:
            return f.read().strip()
    except OSError:
        return None


def _calls_stale(version: str) -> bool:
    return _older(CALLS, [os.path.join(CSRC, CALLS_SOURCE), os.path.join(INCLUDE, "a2cid2.h")]) or calls_version() != version


def _build_calls(tmp: str) -> subprocess.Popen:
    """Starts the build of the host side of the usual operator calls (csrc/torch_calls.cpp), which is linked to torch and to LIB."""
    import torch

    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    include = os.path.join(os.path.dirname(torch.__file__), "include")
    cmd = [shutil.which("g++") or "g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-o", tmp,
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I", INCLUDE, "-isystem", include, "-isystem", os.path.join(include, "torch", "csrc", "api", "include"),
           "-isystem", os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include"), "-isystem", sysconfig.get_paths()["include"],
           os.path.join(CSRC, CALLS_SOURCE), "-L", HERE, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN",
           "-L", lib, "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def _build_library(verbose: bool) -> None:
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
           "-Xcompiler", "-fPIC,-O2,-Wall", "-shared", "-cudart", "static", "--threads", "0",  # sources side by side
           "--diag-error", "2809",  # a launch whose status is dropped ([[nodiscard]])
           "-I", INCLUDE, "-I", CSRC, "-o", tmp]
    cmd += os.environ.get("A2CID2_NVCC_FLAGS", "").split()  # extra flags for experiments, e.g. -DA2_EVENT_THREADS=512
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("nvcc failed")
    if verbose:
        sys.stderr.write(r.stdout + r.stderr)
    os.replace(tmp, LIB)


def build(force: bool = False, verbose: bool = False) -> str:
    """Builds what is missing or older than its sources, and returns the library's path."""
    if force or _stale():
        _build_library(verbose)
    version = torch_version()
    if version is not None and (force or _calls_stale(version)):
        tmp = CALLS + f".tmp{os.getpid()}"
        calls = _build_calls(tmp)
        text = calls.communicate()[0]
        if calls.returncode != 0:
            sys.stderr.write(text)
            raise RuntimeError("g++ failed")
        os.replace(tmp, CALLS)
        with open(tmp + ".torch", "w") as f:
            f.write(version + "\n")
        os.replace(tmp + ".torch", CALLS + ".torch")  # others may be reading it
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
