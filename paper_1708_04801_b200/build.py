"""Builds libwpsgd.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and _rows.so (the Python entry of the operators on
whole sets of rows) with the host compiler."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libwpsgd.so")
BINDING = os.path.join(HERE, "_rows.so")
BINDING_SOURCE = os.path.join(CSRC, "rows_binding.cpp")
OBJ = os.path.join(HERE, "_build")
SOURCES = ["wpsgd_api.cu", "wpsgd_rows.cu"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _newest_source_mtime() -> float:
    m = 0.0
    for root in (CSRC, os.path.join(os.path.dirname(HERE), "include")):
        for f in os.listdir(root):
            if f.endswith((".cu", ".cuh", ".h")):
                m = max(m, os.path.getmtime(os.path.join(root, f)))
    return m


def _fresh(obj: str) -> bool:
    """Whether an object file is newer than every file that its last compilation read (nvcc wrote the list beside it)."""
    try:
        text = open(obj + ".d").read()
        made = os.path.getmtime(obj)
        read = text.split(":", 1)[1].replace("\\\n", " ").split()
        return all(os.path.getmtime(f) <= made for f in read)
    except (OSError, IndexError):
        return False


def _binding_stamp() -> str:
    """What _rows.so is built for beside its sources, and carries: it uses torch's C++ classes and Python's C API."""
    import importlib.metadata
    import sysconfig

    return f"torch {importlib.metadata.version('torch')} python {sysconfig.get_config_var('SOABI')}"


def _binding_fresh() -> bool:
    read = (BINDING_SOURCE, os.path.join(os.path.dirname(HERE), "include", "wpsgd.h"))
    try:
        return all(os.path.getmtime(BINDING) >= os.path.getmtime(f) for f in read) and _binding_stamp().encode() in open(BINDING, "rb").read()
    except OSError:
        return False


def build_binding(force: bool = False) -> str:
    """_rows.so, which calls libwpsgd.so beside it; has to be built after it."""
    if not force and _binding_fresh():
        return BINDING
    import sysconfig

    from torch.utils import cpp_extension

    tmp = BINDING + f".tmp{os.getpid()}"
    include = cpp_extension.include_paths() + [sysconfig.get_paths()["include"], os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include")]
    libs = cpp_extension.library_paths()
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", f'-DROWS_BUILT_FOR="{_binding_stamp()}"', "-o", tmp, BINDING_SOURCE]
                          + [f"-I{i}" for i in include] + [f"-L{i}" for i in libs]
                          + ["-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python", f"-L{HERE}", "-l:libwpsgd.so", "-Wl,-rpath,$ORIGIN"])
    os.replace(tmp, BINDING)
    return BINDING


def build(force: bool = False, verbose: bool = False) -> str:
    lib = build_library(force, verbose)
    build_binding(force)
    return lib


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest_source_mtime():
        return LIB
    os.makedirs(OBJ, exist_ok=True)
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC",
             "-DWPSGD_BUILD"]  # no fast-math: expf and division must round as written
    if verbose:
        flags = ["-Xptxas", "-v"] + flags
    objs, jobs = [], []
    for s in SOURCES:
        obj = os.path.join(OBJ, s + ".o")
        objs.append(obj)
        if force or not _fresh(obj):
            tmp = obj + f".tmp{os.getpid()}"
            cmd = [_nvcc()] + flags + ["-MD", "-MF", tmp + ".d", "-c", "-o", tmp, os.path.join(CSRC, s)]
            jobs.append((obj, tmp, cmd, subprocess.Popen(cmd)))
    failed = None
    for obj, tmp, cmd, job in jobs:
        if job.wait() != 0:
            failed = failed or subprocess.CalledProcessError(job.returncode, cmd)
        else:
            os.replace(tmp + ".d", obj + ".d")
            os.replace(tmp, obj)
    if failed:
        raise failed
    tmp = LIB + f".tmp{os.getpid()}"
    subprocess.check_call([_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", tmp] + objs)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
