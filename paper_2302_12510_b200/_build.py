"""Builds libdybit.so in-tree with nvcc for sm_100a (no JIT cache, no fallback)."""
from __future__ import annotations

import glob
import os
import shutil
import subprocess

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
LIB_PATH = os.path.join(_PKG, "libdybit.so")
DEBUG_LIB_PATH = os.path.join(_PKG, "libdybit_debug.so")     # the same sources with -DDYBIT_DEBUG_BOUNDS (range checks)
_SOURCES = [os.path.join(_PKG, "csrc", f) for f in ("dybit_lib.cu", "dybit_finetune.cu", "dybit_cache.cu")]
_OBJECTS = os.path.join(_PKG, "build")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-std=c++17", "-O3", "-lineinfo",
    "-Xcompiler", "-fPIC",
]


def _nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found: libdybit.so cannot be built")
    return exe


def _deps():
    return (glob.glob(os.path.join(_PKG, "csrc", "*")) +
            glob.glob(os.path.join(_ROOT, "include", "*.h")))


def _flags(debug_bounds: bool) -> list:
    """The options that decide what the compiler makes of a source."""
    return NVCC_FLAGS + (["-DDYBIT_DEBUG_BOUNDS"] if debug_bounds else [])


def _flags_file(path: str) -> str:
    """Where the options are kept that an object or a library was built with."""
    return os.path.join(_OBJECTS, os.path.basename(path) + ".flags")


def _built_with(path: str, flags: list) -> bool:
    try:
        with open(_flags_file(path)) as f:
            return f.read() == "\n".join(flags)
    except OSError:
        return False


def _record_flags(path: str, flags: list) -> None:
    with open(_flags_file(path), "w") as f:
        f.write("\n".join(flags))


def is_stale(path: str = LIB_PATH) -> bool:
    if not os.path.exists(path) or not _built_with(path, _flags(path == DEBUG_LIB_PATH)):
        return True
    t = os.path.getmtime(path)
    return any(os.path.getmtime(p) > t for p in _deps())


def _object_is_stale(obj: str, flags: list) -> bool:
    """Whether the object was built with other options, or a file that it was compiled from (nvcc's list of dependencies
    beside it) is newer than it."""
    if not _built_with(obj, flags):
        return True
    try:
        t = os.path.getmtime(obj)
        with open(obj + ".d") as f:
            deps = f.read().replace("\\\n", " ").split(":", 1)[1].split()
        return any(os.path.getmtime(p) > t for p in deps)
    except (OSError, IndexError):
        return True


def build_library(force: bool = False, verbose: bool = False, debug_bounds: bool = False) -> str:
    """Compile the CUDA sources into paper_2302_12510_b200/libdybit.so (or, with debug_bounds, into
    libdybit_debug.so: the build whose global stores are range-checked, see DYBIT_CHECK in csrc/dybit_common.cuh).
    The translation units are compiled side by side."""
    out = DEBUG_LIB_PATH if debug_bounds else LIB_PATH
    if not force and not is_stale(out):
        return out
    os.makedirs(_OBJECTS, exist_ok=True)
    options = _flags(debug_bounds)
    flags = options + (["-Xptxas", "-v"] if verbose else []) + [
        "-I", os.path.join(_ROOT, "include"), "-I", os.path.join(_PKG, "csrc")]
    objects, jobs = [], []
    for src in _SOURCES:
        obj = os.path.join(_OBJECTS, os.path.basename(src) + (".debug.o" if debug_bounds else ".o"))
        objects.append(obj)
        if force or _object_is_stale(obj, options):
            tmp = obj + ".tmp%d" % os.getpid()
            cmd = [_nvcc()] + flags + ["-c", "-MD", "-MF", obj + ".d", "-o", tmp, src]
            jobs.append((obj, tmp, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    logs = [(obj, tmp, p, p.communicate()[0]) for obj, tmp, p in jobs]
    for obj, tmp, p, log in logs:
        if p.returncode != 0:
            raise RuntimeError("nvcc failed:\n" + log)
        if verbose:
            print(log)
        os.replace(tmp, obj)
        _record_flags(obj, options)
    tmp = out + ".tmp%d" % os.getpid()
    proc = subprocess.run([_nvcc()] + NVCC_FLAGS + ["-shared", "-o", tmp] + objects, capture_output=True, text=True)
    if proc.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + proc.stdout + proc.stderr)
    os.replace(tmp, out)
    _record_flags(out, options)
    return out


if __name__ == "__main__":
    import sys
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv, debug_bounds="--debug-bounds" in sys.argv))
