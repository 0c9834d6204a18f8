"""Build libkforcing.so from csrc/*.cu with nvcc for sm_103a (in-tree), and
_serving.so, the serving operators' Python binding, from csrc/py_serving.cpp
against the installed torch.

Objects go to ``_build/`` next to this file and the shared libraries
beside it.  Translation units compile in parallel; each of the two is skipped when its
sources, flags and compiler (the binding's torch and Python) are unchanged.  The library needs
nvcc alone; where the binding's tools are missing the build says so and leaves it out, and
``serving`` then raises when it is used.
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


def _torch():
    """The installed torch's version and folder (found without importing it), or None."""
    import importlib.metadata
    import importlib.util
    spec = importlib.util.find_spec("torch")
    if spec is None or not spec.origin:
        return None
    return importlib.metadata.version("torch"), os.path.dirname(spec.origin)


def binding_lacks():
    """What the binding cannot be built without and is not here, or None."""
    found = _torch()
    if found is None:
        return "torch"
    if not os.path.exists(os.path.join(found[1], "lib", "libtorch_cuda.so")):
        return "a torch with CUDA"
    if not shutil.which("g++"):
        return "g++"
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        return "Python's headers"
    return None


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


def _digest(names, files) -> str:
    h = hashlib.sha256()
    for x in names:
        h.update(x.encode())
    for f in files + sorted(glob.glob(os.path.join(CSRC, "*.cuh"))) + sorted(glob.glob(os.path.join(ROOT, "include", "*.h"))):
        if os.path.exists(f):
            h.update(f.encode())
            with open(f, "rb") as fh:
                h.update(fh.read())
    return h.hexdigest()


def _stamped(lib, stamp, digest) -> bool:
    if not os.path.exists(lib) or not os.path.exists(stamp):
        return False
    with open(stamp) as f:
        return f.read().strip() == digest


def _compile(nvcc: str, src: str) -> tuple:
    obj = os.path.join(BUILD, os.path.basename(src)[:-3] + ".o")
    cmd = [nvcc, *ARCH, *FLAGS, "-I", os.path.join(ROOT, "include"), "-c", src, "-o", obj]
    p = subprocess.run(cmd, capture_output=True, text=True)
    return obj, p.returncode, p.stdout + p.stderr, cmd


def build(force: bool = False, verbose: bool = False) -> str:
    nvcc = nvcc_path()
    os.makedirs(BUILD, exist_ok=True)
    lacks = binding_lacks()
    stamp, dig = os.path.join(BUILD, "stamp"), _digest(ARCH + FLAGS + [nvcc, os.uname().machine], _sources())
    with_lib = force or not _stamped(LIB, stamp, dig)
    if not lacks:
        binding_stamp, binding_dig = os.path.join(BUILD, "stamp_serving"), _digest([*_torch(), sys.version, os.uname().machine], [BINDING_SRC])
    with_binding = not lacks and (force or not _stamped(BINDING, binding_stamp, binding_dig))
    if lacks:
        sys.stderr.write(f"the serving operators' Python binding (_serving.so) is left out: {lacks} is missing\n")
    srcs = _sources() if with_lib else []
    objs = []
    with cf.ThreadPoolExecutor(max_workers=min(len(srcs) + 1, os.cpu_count() or 4)) as ex:
        binding = ex.submit(_compile_binding, nvcc) if with_binding else None
        for obj, rc, log, cmd in ex.map(lambda s: _compile(nvcc, s), srcs):
            with open(obj + ".log", "w") as f:
                f.write(" ".join(cmd) + "\n" + log)
            if rc != 0:
                sys.stderr.write(log)
                raise RuntimeError("nvcc failed: " + " ".join(cmd))
            if verbose:
                sys.stderr.write(log)
            objs.append(obj)
        if with_binding:
            binding_obj, rc, log, cmd = binding.result()
            if rc != 0:
                sys.stderr.write(log)
                raise RuntimeError("g++ failed: " + " ".join(cmd))
    if with_lib:
        tmp = LIB + ".tmp"
        cmd = [nvcc, *ARCH, "-shared", "-o", tmp, *objs, "-cudart", "static"]
        p = subprocess.run(cmd, capture_output=True, text=True)
        if p.returncode != 0:
            sys.stderr.write(p.stdout + p.stderr)
            raise RuntimeError("link failed: " + " ".join(cmd))
        os.replace(tmp, LIB)
        with open(stamp, "w") as f:
            f.write(dig)
    if with_binding:
        _link_binding(binding_obj)
        with open(binding_stamp, "w") as f:
            f.write(binding_dig)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
