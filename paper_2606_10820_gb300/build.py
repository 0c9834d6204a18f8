"""Build libkforcing.so from csrc/*.cu with nvcc for sm_103a (in-tree), and
_serving.so, the serving operators' Python binding, from csrc/py_serving.cpp
against the installed torch.

Objects go to ``_build/`` next to this file and the shared libraries
beside it.  Translation units compile in parallel; the
build is skipped when the sources, flags, compiler and torch are unchanged.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import hashlib
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libkforcing.so")
BINDING = os.path.join(HERE, "_serving.so")
BINDING_SRC = os.path.join(CSRC, "py_serving.cpp")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-O2",
         "--expt-relaxed-constexpr", "-Xptxas", "-v"]


def nvcc_path() -> str:
    p = shutil.which("nvcc")
    if p:
        return p
    for cand in ("/usr/local/cuda/bin/nvcc",):
        if os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found; the CUDA toolkit is required to build libkforcing.so")


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _torch() -> tuple:
    """The installed torch's version and folder (found without importing it)."""
    import importlib.metadata
    import importlib.util
    spec = importlib.util.find_spec("torch")
    if spec is None or not spec.origin:
        raise RuntimeError("torch is required to build the serving operators' binding")
    return importlib.metadata.version("torch"), os.path.dirname(spec.origin)


def _compile_binding(nvcc: str) -> tuple:
    """py_serving.cpp to an object (of its own suffix: only the library's objects are *.o)."""
    root = _torch()[1]
    obj = os.path.join(BUILD, "py_serving.obj")
    inc = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
           os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include"), sysconfig.get_paths()["include"]]
    cmd = ["g++", "-std=c++17", "-O2", "-fPIC", "-DNDEBUG", *[x for i in inc for x in ("-isystem", i)], "-c", BINDING_SRC, "-o", obj]
    p = subprocess.run(cmd, capture_output=True, text=True)
    return obj, p.returncode, p.stdout + p.stderr, cmd


def _link_binding(obj: str) -> None:
    lib = os.path.join(_torch()[1], "lib")
    tmp = BINDING + ".tmp"
    cmd = ["g++", "-shared", "-o", tmp, obj, "-L", HERE, "-l:libkforcing.so", "-L", lib, "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python",
           "-Wl,-rpath,$ORIGIN", "-Wl,-rpath," + lib]
    p = subprocess.run(cmd, capture_output=True, text=True)
    if p.returncode != 0:
        sys.stderr.write(p.stdout + p.stderr)
        raise RuntimeError("link failed: " + " ".join(cmd))
    os.replace(tmp, BINDING)


def _digest(nvcc: str) -> str:
    h = hashlib.sha256()
    h.update(" ".join(ARCH + FLAGS).encode())
    h.update(nvcc.encode())
    h.update(os.uname().machine.encode())
    h.update((_torch()[0] + sys.version).encode())
    for f in _sources() + [BINDING_SRC] + sorted(glob.glob(os.path.join(CSRC, "*.cuh"))) + \
            sorted(glob.glob(os.path.join(ROOT, "include", "*.h"))):
        if os.path.exists(f):
            h.update(f.encode())
            with open(f, "rb") as fh:
                h.update(fh.read())
    return h.hexdigest()


def _compile(nvcc: str, src: str) -> tuple:
    obj = os.path.join(BUILD, os.path.basename(src)[:-3] + ".o")
    cmd = [nvcc, *ARCH, *FLAGS, "-I", os.path.join(ROOT, "include"), "-c", src, "-o", obj]
    p = subprocess.run(cmd, capture_output=True, text=True)
    return obj, p.returncode, p.stdout + p.stderr, cmd


def build(force: bool = False, verbose: bool = False) -> str:
    nvcc = nvcc_path()
    os.makedirs(BUILD, exist_ok=True)
    stamp = os.path.join(BUILD, "stamp")
    dig = _digest(nvcc)
    if not force and os.path.exists(LIB) and os.path.exists(BINDING) and os.path.exists(stamp):
        with open(stamp) as f:
            if f.read().strip() == dig:
                return LIB
    srcs = _sources()
    objs = []
    with cf.ThreadPoolExecutor(max_workers=min(len(srcs) + 1, os.cpu_count() or 4)) as ex:
        binding = ex.submit(_compile_binding, nvcc)
        for obj, rc, log, cmd in ex.map(lambda s: _compile(nvcc, s), srcs):
            with open(obj + ".log", "w") as f:
                f.write(" ".join(cmd) + "\n" + log)
            if rc != 0:
                sys.stderr.write(log)
                raise RuntimeError("nvcc failed: " + " ".join(cmd))
            if verbose:
                sys.stderr.write(log)
            objs.append(obj)
        binding_obj, rc, log, cmd = binding.result()
        if rc != 0:
            sys.stderr.write(log)
            raise RuntimeError("g++ failed: " + " ".join(cmd))
    tmp = LIB + ".tmp"
    cmd = [nvcc, *ARCH, "-shared", "-o", tmp, *objs, "-cudart", "static"]
    p = subprocess.run(cmd, capture_output=True, text=True)
    if p.returncode != 0:
        sys.stderr.write(p.stdout + p.stderr)
        raise RuntimeError("link failed: " + " ".join(cmd))
    os.replace(tmp, LIB)
    _link_binding(binding_obj)
    with open(stamp, "w") as f:
        f.write(dig)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
