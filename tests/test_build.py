"""What `build()` needs and when it builds again, with stand-ins for the compilers in a copy of the package."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = "paper_2509_23410_b200"
COMPILER = """#!/bin/sh
# a stand-in: notes its name and writes the defines to what it was asked to write
echo "$0" >> "$(dirname "$0")/calls"
text=
while [ $# -gt 0 ]; do
  case "$1" in -o) out="$2"; shift;; -DPATCH_BUILT=*) text="${1#-DPATCH_BUILT=}";; esac
  shift
done
text="${text#\\"}"
printf '%s\\0' "${text%\\"}" > "$out"
"""


@pytest.fixture
def tree(tmp_path):
    pkg = tmp_path / PKG
    (pkg / "csrc").mkdir(parents=True)
    (pkg / "__init__.py").write_text("")
    shutil.copy(os.path.join(ROOT, PKG, "build.py"), pkg)
    shutil.copytree(os.path.join(ROOT, "include"), tmp_path / "include")
    for f in os.listdir(os.path.join(ROOT, PKG, "csrc")):
        shutil.copy(os.path.join(ROOT, PKG, "csrc", f), pkg / "csrc")
    for name in ("nvcc", "g++"):
        (tmp_path / name).write_text(COMPILER)
        (tmp_path / name).chmod(0o755)

    def build(before="pass", **env):
        """Runs build() there; the compilers it called, in order."""
        calls = tmp_path / "calls"
        calls.write_text("")
        code = f"import sys; {before}; from {PKG} import build; print(build.build())"
        r = subprocess.run([sys.executable, "-c", code], cwd=tmp_path, capture_output=True, text=True,
                           env=dict(os.environ, NVCC=str(tmp_path / "nvcc"), **{"CXX": str(tmp_path / "g++"), **env}))
        assert r.returncode == 0, r.stderr
        assert r.stdout.strip() == str(pkg / "libpatch_b200.so") and (pkg / "libpatch_b200.so").exists()
        return [os.path.basename(c) for c in calls.read_text().split()], r.stderr
    build.marshal = pkg / "_marshal.so"
    return build


def test_the_library_needs_no_torch(tree):
    calls, err = tree("sys.modules['torch'] = None")
    assert calls == ["nvcc"] and "was not built" in err and not tree.marshal.exists()


@pytest.mark.parametrize("cxx", ["/bin/false", "/nonexistent/g++"])
def test_nor_a_host_compiler_for_torch(tree, cxx):
    pytest.importorskip("torch")
    calls, err = tree(CXX=cxx)
    assert calls == ["nvcc"] and "was not built" in err


def test_what_is_built_again(tree):
    torch = pytest.importorskip("torch")
    assert tree()[0] == ["nvcc", "g++"]
    assert tree.marshal.read_bytes() == f"for torch {torch.__version__}\0".encode()
    assert tree() == ([], "")
    # the module of another torch, newer than every source
    tree.marshal.write_bytes(f"for torch {torch.__version__}.1\0".encode())
    assert tree()[0] == ["g++"]
    assert tree()[0] == []


def test_a_module_for_another_torch_is_refused(monkeypatch):
    pytest.importorskip("torch")
    from paper_2509_23410_b200 import build
    build.build()
    from paper_2509_23410_b200 import binding as B, _marshal
    B._use_torch()
    monkeypatch.setattr(_marshal, "built", "for torch 1.0")
    with pytest.raises(RuntimeError, match="for torch 1.0"):
        B._use_torch()
