"""Build the CUDA library in-tree with nvcc for sm_100a (no JIT cache, no torch extension)."""

from __future__ import annotations

import os
import shutil
import subprocess
import sys

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
LIB_PATH = os.path.join(PKG_DIR, "libbrace.so")
DEBUG_LIB_PATH = os.path.join(PKG_DIR, "libbrace_debug.so")
OBJ_DIR = os.path.join(PKG_DIR, "_build")
SOURCES = [os.path.join(PKG_DIR, "csrc", f) for f in ("brace.cu", "operators.cu")]
DEPS = SOURCES + [os.path.join(PKG_DIR, "csrc", f) for f in ("brace_kernels.cuh", "elements.cuh", "embedding_kernels.cuh",
                                                            "ortho_kernels.cuh", "sm100.cuh")]
DEPS += [os.path.join(ROOT, "include", "brace.h")]


def _nvcc() -> str:
    cand = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found: the BRACE CUDA library cannot be built")
    return cand


def needs_build(path: str = LIB_PATH) -> bool:
    if not os.path.exists(path):
        return True
    t = os.path.getmtime(path)
    return any(os.path.getmtime(p) > t for p in DEPS)


def _object(source: str, defines) -> str:
    """Where a source's object lies; only brace.cu looks at the defines."""
    name = os.path.splitext(os.path.basename(source))[0]
    if defines and name == "brace":
        name += "_debug"
    return os.path.join(OBJ_DIR, name + ".o")


def _compile(out_path: str, defines, verbose: bool) -> str:
    base = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
            "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG_DIR, "csrc")]
    os.makedirs(OBJ_DIR, exist_ok=True)
    objects, running = [], []
    for source in SOURCES:
        obj = _object(source, defines)
        objects.append(obj)
        if not verbose and not needs_build(obj):
            continue
        # written elsewhere first: an object that is there is whole
        part = f"{obj}.{os.getpid()}.o"
        cmd = base + (["-Xptxas", "-v"] if verbose else []) + list(defines) + ["-c", source, "-o", part]
        running.append((part, obj, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = ""
    for part, obj, proc in running:
        said = proc.communicate()[0]
        if proc.returncode != 0:
            failed += said
            continue
        os.replace(part, obj)
        if verbose:
            sys.stderr.write(said)
    if failed:
        raise RuntimeError("nvcc failed:\n" + failed)
    res = subprocess.run(base + ["-shared", "-o", out_path] + objects, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    return out_path


def _forget_objects(defines) -> None:
    """A forced build compiles anew; the debug library shares what does not look at its define."""
    for source in SOURCES:
        obj = _object(source, defines)
        if os.path.exists(obj) and not (defines and obj == _object(source, [])):
            os.remove(obj)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB_PATH
    if force:
        _forget_objects([])
    return _compile(LIB_PATH, [], verbose)


def build_debug(force: bool = False, verbose: bool = False) -> str:
    """The same library with -DBRACE_DEBUG: ring kernels check their index ranges and report through
    brace_debug_status instead of trapping.  Load it by setting BRACE_LIBRARY to the returned path."""
    if not force and not needs_build(DEBUG_LIB_PATH):
        return DEBUG_LIB_PATH
    if force:
        _forget_objects(["-DBRACE_DEBUG"])
    return _compile(DEBUG_LIB_PATH, ["-DBRACE_DEBUG"], verbose)


if __name__ == "__main__":
    if "--debug" in sys.argv:
        print(build_debug(force="--force" in sys.argv, verbose="-v" in sys.argv))
    else:
        print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
