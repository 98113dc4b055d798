"""Builds libnsml.so in-tree with nvcc for sm_100a (cross-compiles without a GPU), and the module that calls its 8-bit operators
from Python (the rest goes through ctypes).

    python -m paper_2506_16235_b200.build [--force] [--verbose]
"""
from __future__ import annotations

import hashlib
import os
import shutil
import subprocess
import sys
import sysconfig

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB_PATH = os.path.join(PKG_DIR, "libnsml.so")
STAMP_PATH = LIB_PATH + ".stamp"
NATIVE_PATH = os.path.join(PKG_DIR, "_native" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))

SOURCES = ["nsml_api.cu", "nsml_grid_large.cu", "nsml_q8_rows.cu", "nsml_q8_norm_grad.cu", "nsml_q8_gemm.cu", "nsml_q8_tokens.cu", "nsml_controller.cpp"]
FLAGS = [
    "-O3", "-std=c++17", "-lineinfo",
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-ftz=false", "-prec-div=true", "-prec-sqrt=true", "-fmad=false",
    "-Xcompiler", "-fPIC", "-Xcompiler", "-ffp-contract=off",
    "-shared", "-cudart", "static", "--threads", "7",
]
NATIVE_SOURCE = "nsml_python.cpp"
NATIVE_FLAGS = ["-O2", "-std=c++17", "-fPIC", "-shared", "-Wall"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found (set NVCC or put it on PATH)")


def _inputs():
    files = [os.path.join(INCLUDE, "nsml.h")]
    for name in sorted(os.listdir(CSRC)):
        if name.endswith((".cu", ".cuh", ".cpp", ".h")):
            files.append(os.path.join(CSRC, name))
    return files


def _fingerprint() -> str:
    h = hashlib.sha256()
    for f in _inputs():
        h.update(os.path.basename(f).encode())
        with open(f, "rb") as fh:
            h.update(fh.read())
    h.update(" ".join(FLAGS + NATIVE_FLAGS).encode())
    return h.hexdigest()


def _library_is_stale() -> bool:
    if not (os.path.exists(LIB_PATH) and os.path.exists(STAMP_PATH)):
        return True
    with open(STAMP_PATH) as fh:
        return fh.read().strip() != _fingerprint()


def is_stale() -> bool:
    """True if the library or the module is missing or was built from other sources or flags
    (content hash, so file times do not matter)."""
    return _library_is_stale() or not os.path.exists(NATIVE_PATH)


def _cxx() -> str:
    for cand in (os.environ.get("CXX"), shutil.which("g++"), shutil.which("c++")):
        if cand and shutil.which(cand):
            return cand
    raise RuntimeError("no C++ compiler found (set CXX or put g++ on PATH)")


def _run(cmd, what: str, verbose: bool) -> None:
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
    if res.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed building {what}")


def build_native(verbose: bool = False) -> None:
    """The Python module, linked to the library next to it."""
    tmp = NATIVE_PATH + ".tmp"
    _run([_cxx()] + NATIVE_FLAGS + ["-I", INCLUDE, "-I", sysconfig.get_paths()["include"], os.path.join(CSRC, NATIVE_SOURCE), "-o", tmp,
                                    "-L", PKG_DIR, "-l:" + os.path.basename(LIB_PATH), "-Wl,-rpath,$ORIGIN"], os.path.basename(NATIVE_PATH), verbose)
    os.replace(tmp, NATIVE_PATH)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile the library and the module if they are missing or older than their sources."""
    if not force and not _library_is_stale():
        if not os.path.exists(NATIVE_PATH):
            build_native(verbose)
        return LIB_PATH
    cmd = [_nvcc()] + FLAGS + ["-I", INCLUDE, "-I", CSRC]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    tmp = LIB_PATH + ".tmp"
    cmd += ["-o", tmp]
    _run(cmd, "libnsml.so", verbose)
    os.replace(tmp, LIB_PATH)
    build_native(verbose)
    with open(STAMP_PATH, "w") as fh:
        fh.write(_fingerprint() + "\n")
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
