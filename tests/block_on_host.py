"""Kernels' own source, compiled for the CPU and run one block at a time
(block_on_host.h): for what a GPU shows only by chance or must not be shown at all."""
import ctypes
import os
import re
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2606_10820_gb300", "csrc")


def between(file, first, end):
    """The source of `file` from the text `first` up to the text `end`, each there once."""
    with open(os.path.join(CSRC, file)) as f:
        text = f.read()
    assert text.count(first) == 1 and text.count(end) == 1, (first, end)
    return text[text.index(first):text.index(end)]


def load(tmp_path, name, source, driver):
    """The kernels' source and C entry points that call block::run, as a library."""
    source = re.sub(r"extern __shared__[^;]*\bsm\[\];", "uint8_t* sm = block::dynamic_shared;", source)
    source = re.sub(r'asm volatile\("griddepcontrol\.[^;]*;" ::: "memory"\);', "", source)
    src, out = os.path.join(tmp_path, name + ".cpp"), os.path.join(tmp_path, name + ".so")
    with open(src, "w") as f:
        f.write('#include "block_on_host.h"\n#include "kforcing_serving.h"\n' + source + driver)
    p = subprocess.run(["g++", "-std=c++17", "-O1", "-fwrapv", "-w", "-shared", "-fPIC", "-I", HERE,
                        "-I", os.path.join(os.path.dirname(HERE), "include"), "-o", out, src], capture_output=True, text=True)
    assert p.returncode == 0, p.stderr
    return ctypes.CDLL(out)


def orders(warps=32):
    """Ascending, descending, and the first warp behind all others."""
    up = list(range(warps))
    return [(ctypes.c_int * warps)(*x) for x in (up, up[::-1], up[1:] + up[:1])]
