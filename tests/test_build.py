"""What a build needs: libkforcing.so the CUDA compiler alone, the serving operators' binding torch and
a C++ compiler too (a compiler that writes empty files stands in)."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
COMPILER = """#!/bin/sh
echo "$0 $*" >> "$LOG"
while [ $# -gt 0 ]; do
  if [ "$1" = -o ]; then : > "$2"; fi
  shift
done
"""


@pytest.fixture
def tree(tmp_path):
    """A copy of what build.py reads, and folders with stand-ins for nvcc and g++."""
    pkg = "paper_2606_10820_gb300"
    shutil.copytree(os.path.join(ROOT, "include"), tmp_path / "tree" / "include")
    shutil.copytree(os.path.join(ROOT, pkg, "csrc"), tmp_path / "tree" / pkg / "csrc")
    shutil.copy(os.path.join(ROOT, pkg, "build.py"), tmp_path / "tree" / pkg / "build.py")
    for name in ("nvcc", "g++"):
        (tmp_path / name / "bin").mkdir(parents=True)
        f = tmp_path / name / "bin" / name
        f.write_text(COMPILER)
        f.chmod(0o755)

    def build(*flags, tools=("nvcc", "g++"), also=""):
        path = ":".join(str(tmp_path / t / "bin") for t in tools)
        log = tmp_path / "log"
        log.write_text("")
        p = subprocess.run([sys.executable, *flags, "-c", "import sys; sys.path.insert(0, sys.argv[1]); import build; " + also + "print(build.build())",
                            str(tmp_path / "tree" / pkg)], capture_output=True, text=True, env={"PATH": path, "LOG": str(log)})
        return p, log.read_text(), tmp_path / "tree" / pkg

    return build


@pytest.mark.parametrize("flags,tools,why", [(["-S"], ("nvcc", "g++"), "torch"), ([], ("nvcc",), "g++")])
def test_the_library_needs_neither_torch_nor_the_binding(tree, flags, tools, why):
    """-S: without the installed packages."""
    p, log, pkg = tree(*flags, tools=tools)
    assert p.returncode == 0, p.stderr
    assert p.stdout.strip() == str(pkg / "libkforcing.so") and (pkg / "libkforcing.so").exists()
    assert not (pkg / "_serving.so").exists() and "_serving" in p.stderr and why in p.stderr
    # nothing is compiled again
    p, log, _ = tree(*flags, tools=tools)
    assert p.returncode == 0 and log == ""


def test_the_binding_follows_when_torch_is_there(tree):
    pytest.importorskip("torch")
    enough = "build.binding_lacks = lambda: None; "      # (this machine's torch, whatever it was built for)
    assert tree("-S")[0].returncode == 0
    p, log, pkg = tree(also=enough)
    assert p.returncode == 0, p.stderr
    assert (pkg / "_serving.so").exists() and "nvcc/bin/nvcc" not in log and "py_serving.cpp" in log
    assert tree(also=enough)[1] == ""
    # the binding alone, and the library alone
    (pkg / "_serving.so").unlink()
    assert "nvcc/bin/nvcc" not in tree(also=enough)[1] and (pkg / "_serving.so").exists()
    (pkg / "libkforcing.so").unlink()
    log = tree(also=enough)[1]
    assert "nvcc/bin/nvcc" in log and (pkg / "libkforcing.so").exists()


def test_a_binding_that_does_not_compile_is_an_error(tree, tmp_path):
    pytest.importorskip("torch")
    (tmp_path / "g++" / "bin" / "g++").write_text("#!/bin/sh\nexit 1\n")
    p, _, pkg = tree(also="build.binding_lacks = lambda: None; ")
    assert p.returncode != 0 and "g++ failed" in p.stderr and not (pkg / "_serving.so").exists()
