"""Build step: compiles the CUDA sources under csrc/ into libharp.so (sm_100a only) and csrc/pycall.c into
_harpcall.abi3.so (the call from Python; ctypes does without it), in-tree, next to this file.  ``python -m paper_2605_29843_b200.build`` or build()."""
from __future__ import annotations

import fcntl
import glob
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libharp.so")
OBJECTS = os.path.join(HERE, "_build")
CALL, CALL_SRC = os.path.join(HERE, "_harpcall.abi3.so"), os.path.join(HERE, "csrc", "pycall.c")


def sources():
    return sorted(glob.glob(os.path.join(HERE, "csrc", "*.cu")))


def headers_of_sources():
    return glob.glob(os.path.join(HERE, "csrc", "*.h")) + glob.glob(os.path.join(HERE, "csrc", "*.cuh")) \
        + glob.glob(os.path.join(ROOT, "include", "*.h"))


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + headers_of_sources()
    return any(os.path.getmtime(p) > t for p in deps)


def _call_stale() -> bool:
    return (not os.path.exists(CALL) or os.path.getmtime(CALL_SRC) > os.path.getmtime(CALL)) and \
        os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h"))


def _produce(cmd, target) -> None:
    """What a command that was interrupted leaves is never taken for its result."""
    part = os.path.join(OBJECTS, os.path.basename(target) + ".part")
    subprocess.check_call(cmd + ["-o", part])
    os.replace(part, target)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale() and not _call_stale():
        return LIB
    os.makedirs(OBJECTS, exist_ok=True)
    with open(os.path.join(OBJECTS, "lock"), "w") as lock:        # one build of a tree at a time
        fcntl.flock(lock, fcntl.LOCK_EX)
        if force or _call_stale():
            headers = sysconfig.get_paths()["include"]
            if os.path.exists(os.path.join(headers, "Python.h")):
                _produce([os.environ.get("CC", "gcc"), "-shared", "-fPIC", "-O2", "-I", headers, CALL_SRC], CALL)
        if force or _stale():
            _build_lib(force, verbose)
    return LIB


def _build_lib(force: bool, verbose: bool) -> None:
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-c", "-Xcompiler", "-fPIC", "-std=c++17", "-O3", "-lineinfo",
           "-gencode", "arch=compute_100a,code=sm_100a",
           "-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "csrc")]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    if os.environ.get("HARP_TM_TIMING"):          # per-section cycle counters in the tensor-memory kernels
        cmd += ["-DHARP_TM_TIMING"]
    if os.environ.get("HARP_FAST_TIMING"):        # ... and in the whole-row kernel
        cmd += ["-DHARP_FAST_TIMING"]
    # An object a source: several at a time, and those alone whose source or headers changed.  Kept objects belong to the command and the
    # compiler that the key names; it is gone while some may be of another one.
    headers_at = max(os.path.getmtime(p) for p in headers_of_sources())
    key_at, key = os.path.join(OBJECTS, "command"), repr(cmd) + subprocess.check_output([nvcc, "--version"], text=True)
    if os.path.exists(key_at):
        with open(key_at) as f:
            force |= f.read() != key
    else:
        force = True
    if force and os.path.exists(key_at):
        os.remove(key_at)

    def compile_one(src):
        obj = os.path.join(OBJECTS, os.path.basename(src) + ".o")
        if force or not os.path.exists(obj) or os.path.getmtime(obj) < max(headers_at, os.path.getmtime(src)):
            _produce(cmd + [src], obj)
        return obj

    with ThreadPoolExecutor(os.cpu_count() or 1) as pool:
        objects = list(pool.map(compile_one, sources()))
    with open(key_at, "w") as f:
        f.write(key)
    _produce([nvcc, "-shared", "-gencode", "arch=compute_100a,code=sm_100a", *objects], LIB)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
