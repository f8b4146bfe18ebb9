"""Builds libcovspec.so in-tree with nvcc for sm_100a (no torch extension machinery: the library
is a plain C ABI loaded through ctypes), and the native part of the Python binding with g++ against torch's headers."""
from __future__ import annotations

import hashlib
import os
import re
import subprocess
import sys
import sysconfig
import time

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcovspec.so")
LIB_DEBUG = os.path.join(HERE, "libcovspec_debug.so")     # the same sources with -DCOVSPEC_DEBUG_BOUNDS
OBJECTS = os.path.join(HERE, "_build")                    # a compiled source is used again until one of its files, its command or the
                                                          # compiler changes
SOURCES = ["covspec.cu", "verify.cu", "attend_bf16.cu", "attend_f16.cu"]
BINDING_SOURCE = os.path.join(CSRC, "binding.cpp")


def _newest(paths):
    return max(os.path.getmtime(p) for p in paths)


def _files_of(source: str) -> list:
    """The source and what it includes of this library."""
    found, todo = [], [source]
    while todo:
        path = todo.pop()
        if path in found:
            continue
        found.append(path)
        with open(path) as f:
            names = re.findall(r'^\s*#include "([^"]+)"', f.read(), re.M)
        todo += [p for n in names for p in (os.path.join(CSRC, n), os.path.join(ROOT, "include", n)) if os.path.exists(p)]
    return found


def binding_path() -> str:
    """The native part of the binding holds to one Python and one torch, which its name gives: another one does not find
    it and builds its own."""
    import torch
    return os.path.join(HERE, f"_binding.{sys.implementation.cache_tag}.torch-{torch.__version__}.so")


def needs_build(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return True
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != os.path.basename(BINDING_SOURCE)] + \
           [os.path.join(ROOT, "include", "covspec.h")]
    return _newest(deps) > os.path.getmtime(lib)


def build(force: bool = False, verbose: bool = False, debug_bounds: bool = False) -> str:
    """Builds the library if a source is newer than it.  debug_bounds=True builds the checked variant
    (libcovspec_debug.so): index-driven accesses test their index and report COVSPEC_ERR_BOUNDS.
    The native part of the binding is built too; where that fails (no Python headers) the library is complete without
    it, its calls go through ctypes."""
    if not debug_bounds:
        try:
            build_binding(force)
        except (RuntimeError, OSError) as e:
            sys.stderr.write(f"the native part of the binding was not built, calls will go through ctypes: {e}\n")
    LIB = LIB_DEBUG if debug_bounds else globals()["LIB"]
    if not force and not needs_build(LIB):
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    target = ["-gencode", "arch=compute_100a,code=sm_100a"]
    common = [nvcc, "-c", "-Xcompiler", "-fPIC", "-O3", "-std=c++17", "-lineinfo", *target,
              "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    if debug_bounds:
        common.append("-DCOVSPEC_DEBUG_BOUNDS")
    os.makedirs(OBJECTS, exist_ok=True)
    # objects of another command or compiler are not linked with these
    version = subprocess.run([nvcc, "--version"], capture_output=True, text=True).stdout
    key = hashlib.sha256("\0".join([*common, version]).encode()).hexdigest()[:12]
    objects, running = [], []
    for name in SOURCES:
        source = os.path.join(CSRC, name)
        objects.append(os.path.join(OBJECTS, f"{os.path.splitext(name)[0]}{'_debug' if debug_bounds else ''}-{key}.o"))
        # verbose: what the compiler says of every source
        if force or verbose or not os.path.exists(objects[-1]) or _newest(_files_of(source)) > os.path.getmtime(objects[-1]):
            # under a name of its own until it is whole: what is there later is complete
            part = f"{objects[-1]}.{os.getpid()}.part"
            began = time.time()
            running.append((objects[-1], part, began, subprocess.Popen([*common, *(["-Xptxas", "-v"] if verbose else []), "-o", part, source],
                                                                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = False
    for path, part, began, job in running:
        said = job.communicate()[0]
        failed |= job.returncode != 0
        if job.returncode or verbose:
            sys.stderr.write(said)
        if not job.returncode:
            os.utime(part, (began, began))            # a file that changes while it is read is newer than what was made of it
            os.replace(part, path)
    if not failed:
        res = subprocess.run([nvcc, "-shared", "-Xcompiler", "-fPIC", *target, "-o", LIB, *objects], capture_output=True, text=True)
        failed = res.returncode != 0
        if failed:
            sys.stderr.write(res.stdout + res.stderr)
    if failed:
        raise RuntimeError("nvcc failed building " + os.path.basename(LIB))
    return LIB


def build_binding(force: bool = False) -> str:
    import torch
    target = binding_path()
    if not force and os.path.exists(target) and _newest(_files_of(BINDING_SOURCE)) <= os.path.getmtime(target):
        return target
    base = os.path.dirname(torch.__file__)
    libs = os.path.join(base, "lib")
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-shared", "-fPIC", "-std=c++17",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I", os.path.join(base, "include"), "-I", os.path.join(base, "include", "torch", "csrc", "api", "include"),
           "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"], "-I", os.path.join(cuda, "include"),
           "-o", target, BINDING_SOURCE, "-L", libs, "-lc10", "-lc10_cuda", "-ltorch", "-ltorch_cpu", "-ltorch_python",
           "-Wl,-rpath," + libs]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("g++ failed building " + os.path.basename(target))
    return target


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv, debug_bounds="--debug-bounds" in sys.argv))
