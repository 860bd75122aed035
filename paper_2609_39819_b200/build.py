"""Builds libkvt.so in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import importlib.metadata
import os
import subprocess
import sysconfig
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libkvt.so")
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC"]
DEFINES: list = []
HEADER = os.path.join(_HERE, "..", "include", "kvt.h")
# The model-side kernels, most of the compiler's time, have no checked or traced parts: one object for all libraries, linked
# together from those of its sources.
ATTEND_OBJ = os.path.join(_HERE, "kvt_attend.o")
ATTEND_SOURCES = [os.path.join(CSRC, f) for f in ("kvt_attend.cu", "kvt_blocks.cu")]
ATTEND_DEPS = ATTEND_SOURCES + [os.path.join(CSRC, f) for f in ("kvt_attend.h", "kvt_attend.cuh")]
TORCH_SOURCE = "kvt_torch.cpp"


def _torch_lib() -> str:
    """The file of the native marshalling. It is built against one torch and one Python, and named after them: another of either
    does not find it."""
    try:
        torch_version = importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:
        torch_version = "none"
    return os.path.join(_HERE, f"_kvt_torch.{torch_version}.{sysconfig.get_config_var('SOABI')}.so")


TORCH_LIB = _torch_lib()


def _older(target: str, files) -> bool:
    return not os.path.exists(target) or any(os.path.getmtime(f) > os.path.getmtime(target) for f in files)


def _stale(lib: str = LIB) -> bool:
    return _older(lib, [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != TORCH_SOURCE] + [HEADER])


def _make(target: str, stale, command, force: bool = False) -> str:
    """Runs command(temporary file) where `target` is stale. Safe when several processes or threads call it at once (one rank per
    GPU): an exclusive file lock serialises them, the compiler writes to a temporary file and the result is moved into place
    in one step, so nobody ever loads a half-written file."""
    if not (force or stale()):
        return target
    import fcntl
    with open(target + ".lock", "w") as lock:
        fcntl.flock(lock, fcntl.LOCK_EX)
        try:
            if force or stale():             # somebody else may have built it while we waited
                tmp = f"{target}.{os.getpid()}.tmp"
                try:
                    command(tmp)
                    os.replace(tmp, target)
                finally:
                    if os.path.exists(tmp):
                        os.remove(tmp)
        finally:
            fcntl.flock(lock, fcntl.LOCK_UN)
    return target


DEBUG_LIB = os.path.join(_HERE, "libkvt_debug.so")


def build_debug_lib(force: bool = False) -> str:
    """The checked build of the same sources (-DKVT_DEBUG): index / invariant checks in the kernels that set the
    device error word, and every launch in another shape (64-thread blocks, a handful of mover CTAs, no CUDA
    graph). Load it with KVT_LIB=<path>. Used by the tests; the product is libkvt.so."""
    return build_lib(force, lib=DEBUG_LIB, defines=["-DKVT_DEBUG"])


def build_lib(force: bool = False, verbose: bool = False, lib: str = LIB, defines=None) -> str:
    """Compiles libkvt.so if it is missing or older than its sources (several processes may ask at once)."""
    nvcc = [os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")] + NVCC_FLAGS + DEFINES + (["-Xptxas", "-v"] if verbose else [])

    def attend_object(tmp):
        parts = [f"{tmp}.{i}.o" for i in range(len(ATTEND_SOURCES))]
        try:
            with ThreadPoolExecutor(len(parts)) as each:
                for done in [each.submit(subprocess.check_call, nvcc + ["-c", "-o", part, src]) for part, src in zip(parts, ATTEND_SOURCES)]:
                    done.result()
            subprocess.check_call(["ld", "-r", "-o", tmp] + parts)
        finally:
            for part in parts:
                if os.path.exists(part):
                    os.remove(part)

    def attend():
        return _make(ATTEND_OBJ, lambda: _older(ATTEND_OBJ, ATTEND_DEPS), attend_object, force and lib == LIB)

    def link(tmp):
        engine = tmp + ".engine.o"
        with ThreadPoolExecutor(1) as other:         # both sources at once
            obj = other.submit(attend)
            try:
                subprocess.check_call(nvcc + list(defines or []) + ["-c", "-o", engine, os.path.join(CSRC, "kvt_engine.cu")])
                subprocess.check_call(nvcc + ["-shared", "-o", tmp, engine, obj.result()])
            finally:
                if os.path.exists(engine):
                    os.remove(engine)

    return _make(lib, lambda: _stale(lib), link, force)


TRACE_LIB = os.path.join(_HERE, "libkvt_trace.so")


def build_trace_lib(force: bool = False) -> str:
    """Development build with per-kernel event timing (-DKVT_TRACE): with KVT_TRACE=1 in the environment the LOOKUP
    and selection calls print the time between their launches to stderr; KVT_NO_OVERLAP=1 launches the LOOKUP kernels
    without the tail overlap, KVT_NO_GRAPH=1 the selection without its CUDA graph. Load it with KVT_LIB=<path>."""
    return build_lib(force, lib=TRACE_LIB, defines=["-DKVT_TRACE"])


def _cuda_home() -> str:
    return os.environ.get("CUDA_HOME") or os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))


def build_torch_lib(force: bool = False) -> str:
    """The native marshalling of append_kv and attend (a CPython module against torch's headers), compiled with g++ if it is
    missing or older than its source (several processes may ask at once)."""
    src = os.path.join(CSRC, TORCH_SOURCE)

    def compile_(tmp):
        import torch
        at = os.path.dirname(torch.__file__)
        subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC",
                               f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I" + os.path.join(at, "include"),
                               "-I" + os.path.join(at, "include", "torch", "csrc", "api", "include"),
                               "-I" + sysconfig.get_paths()["include"], "-I" + os.path.join(_cuda_home(), "include"), "-o", tmp, src,
                               "-L" + os.path.join(at, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"])

    return _make(TORCH_LIB, lambda: _older(TORCH_LIB, [src, HEADER]), compile_, force)


def build_all() -> None:
    """Every library of the package, compiled side by side."""
    with ThreadPoolExecutor(4) as pool:
        for done in [pool.submit(f) for f in (build_lib, build_torch_lib, build_debug_lib, build_trace_lib)]:
            done.result()


if __name__ == "__main__":
    import sys
    if "--trace" in sys.argv:
        print(build_trace_lib(force=True))
    else:
        print(build_lib(force=True, verbose="-v" in sys.argv))
        print(build_torch_lib(force=True))
