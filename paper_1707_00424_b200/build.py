"""Build libparle.so (sm_100a) with nvcc and the token operators' Python module _token_ops.so with g++, both in-tree."""
from __future__ import annotations

import contextlib
import fcntl
import hashlib
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libparle.so")
MODULE = os.path.join(HERE, "_token_ops.so")
SOURCES = ["parle_api.cu", "static_loss.cu", "token_logprobs.cu", "embedding.cu", "dropout.cu"]
HEADERS = ["common.cuh", "mlp_simt.cuh", "umma_gemm.cuh", "umma_pair_gemm.cuh", "umma_wgrad_update.cuh", "umma_tf32x3.cuh", "update_kernels.cuh", "token_types.cuh"]


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the Parle CUDA library cannot be built")


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS]
    deps.append(os.path.join(HERE, "..", "include", "parle.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def _run(cmd) -> str:
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"{os.path.basename(cmd[0])} failed:\n" + res.stdout + res.stderr)
    return res.stderr


def _compile(cmd, target: str) -> str:
    """Run a compiler for `target`, which changes at once and only when the whole of it is there."""
    part = f"{target[:-len('.so')]}.{os.getpid()}.so"
    try:
        log = _run(cmd + ["-o", part])
        os.replace(part, target)
    finally:
        if os.path.exists(part):
            os.remove(part)
    return log


@contextlib.contextmanager
def _one_at_a_time():
    """Of the processes that build (ranks started together on a fresh tree), one builds and the others wait."""
    fd = os.open(HERE, os.O_RDONLY)
    try:
        fcntl.flock(fd, fcntl.LOCK_EX)
        yield
    finally:
        os.close(fd)


def _compile_library(verbose: bool = False) -> None:
    cmd = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "--threads", "0",
           "-shared", "-Xcompiler", "-fPIC"] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    log = _compile(cmd, LIB)
    if verbose:
        print(log)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile the library if it is missing or older than its sources; return its path."""
    if force or _stale():
        with _one_at_a_time():
            if force or _stale():
                _compile_library(verbose)
    return LIB


MODULE_SOURCES = [os.path.join(CSRC, "token_bindings.cpp"), os.path.join(HERE, "..", "include", "parle.h")]


def module_stamp() -> str:
    """What the module has to be built from: the torch and the Python that are running and its sources' contents (nothing behind "of " where
    there are only built files).  The compiler puts it into the module, so that one built from anything else is known whatever the
    files' times are."""
    import torch
    stamp = f"token operators for torch {torch.__version__}, {sys.implementation.cache_tag}, of "
    if not all(os.path.exists(path) for path in MODULE_SOURCES):
        return stamp
    h = hashlib.sha256()
    for path in MODULE_SOURCES:
        with open(path, "rb") as f:
            h.update(f.read())
    return stamp + h.hexdigest()[:32]


def _module_stale() -> bool:
    if not os.path.exists(MODULE):
        return True
    with open(MODULE, "rb") as f:
        return module_stamp().encode() not in f.read()


def _compile_module() -> None:
    import torch
    at = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(_nvcc())))
    _compile([shutil.which("g++") or "c++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
              f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DBUILT_FROM="{module_stamp()}"', "-isystem", os.path.join(at, "include"),
              "-isystem", sysconfig.get_paths()["include"], "-isystem", os.path.join(cuda, "include"), os.path.join(CSRC, "token_bindings.cpp"),
              "-L" + HERE, "-l:libparle.so", "-L" + os.path.join(at, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10", "-Wl,-rpath,$ORIGIN"], MODULE)


def build_module(force: bool = False) -> str:
    """Compile the Python module of the token operators, which calls the library beside it, if it is missing or was built from other sources or for
    another torch or Python than the ones here; return its path."""
    if force or _module_stale():
        if not os.path.exists(MODULE_SOURCES[0]):
            raise RuntimeError(f"{MODULE} is missing or not built as \"{module_stamp()}..\", and its sources are not here to build it from")
        with _one_at_a_time():
            if _stale():
                _compile_library()
            if force or _module_stale():
                _compile_module()
    return MODULE


if __name__ == "__main__":
    print(build(force=True, verbose=True))
    print(build_module(force=True))
