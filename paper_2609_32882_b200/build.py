"""Builds the CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB_PATH = os.path.join(HERE, "libvsa2.so")
MARSHAL_PATH = os.path.join(HERE, "_marshal.so")      # CPython module that hands the binding's short calls to the library
ARCH_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a"]


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _older(path, *deps):
    """Whether `path` is missing or older than one of `deps`."""
    return not os.path.exists(path) or any(os.path.getmtime(d) > os.path.getmtime(path) for d in deps)


def _header():
    return os.path.join(ROOT, "include", "vsa2.h")


def _stale():
    return _older(LIB_PATH, *(os.path.join(CSRC, f) for f in os.listdir(CSRC) if not f.endswith(".c")), _header())


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compiles csrc/*.cu into libvsa2.so next to this file, and csrc/marshal.c into _marshal.so; returns the library's path.

    The library stands without the module (attention, gate, router go through ctypes): where the module cannot be compiled, say without Python's
    headers, that is said on stderr and the calls that need it fail (binding._marshal)."""
    if force or _stale():
        _build_cuda(force, verbose)
    if force or _older(MARSHAL_PATH, os.path.join(CSRC, "marshal.c"), _header()):
        _build_marshal()
    return LIB_PATH


def _build_marshal():
    if os.path.exists(MARSHAL_PATH):
        os.remove(MARSHAL_PATH)      # (of another header's structs)
    try:
        subprocess.run([shutil.which("gcc") or "cc", "-shared", "-fPIC", "-O2", "-I", sysconfig.get_paths()["include"], "-I", os.path.join(ROOT, "include"),
                        os.path.join(CSRC, "marshal.c"), "-o", MARSHAL_PATH], check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    except (OSError, subprocess.CalledProcessError) as e:
        said = (getattr(e, "output", None) or b"").decode(errors="replace")
        sys.stderr.write(f"{said}{os.path.basename(MARSHAL_PATH)} was not built ({e}): the calls between hidden states and attention will fail\n")


def _build_cuda(force, verbose):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    objs = []
    obj_dir = os.path.join(HERE, "build")
    os.makedirs(obj_dir, exist_ok=True)
    common = [nvcc, "-std=c++17", "-O3", "-lineinfo", "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"),
              "-I", CSRC] + ARCH_FLAGS
    if verbose:
        common += ["-Xptxas", "-v"]
    procs = []
    for src in sources():
        obj = os.path.join(obj_dir, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        hdrs = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cuh")] + [os.path.join(ROOT, "include", "vsa2.h")]
        newest = max(os.path.getmtime(p) for p in [src] + hdrs)
        if not force and os.path.exists(obj) and os.path.getmtime(obj) > newest:
            continue
        procs.append((src, subprocess.Popen(common + ["-c", src, "-o", obj], stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
    for src, pr in procs:
        out, _ = pr.communicate()
        if verbose or pr.returncode:
            sys.stderr.write(out.decode())
        if pr.returncode:
            raise RuntimeError(f"nvcc failed on {src}")
    subprocess.check_call([nvcc, "-shared", "-o", LIB_PATH] + objs + ARCH_FLAGS + ["-lcudart_static", "-ldl", "-lrt", "-lpthread"])


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
