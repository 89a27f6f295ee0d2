"""The policy operators' host side (no GPU needed)."""
from __future__ import annotations

import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2407_04221_gb300 import build
    build.build()


def run(code):
    """Python code in a process of its own: (exit code, output)."""
    p = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    return p.returncode, p.stdout.strip() + p.stderr[-2000:]


def test_scan_sizes_of_nothing():
    """A batch without sequences or channels keeps nothing and works in nothing, however long it is."""
    code = """
import ctypes
import paper_2407_04221_gb300 as av
for T in (0, 1, 4, 100, 1000, 100000):
    for B, D in ((0, 256), (4, 0), (0, 0)):
        for dtype in range(3):
            s, w = ctypes.c_int64(-1), ctypes.c_int64(-1)
            assert av.load().av_scan_sizes(T, B, D, dtype, ctypes.byref(s), ctypes.byref(w)) == 0
            assert s.value == w.value == 0, (T, B, D, dtype, s.value, w.value)
print("all")"""
    assert run(code) == (0, "all")


FAKE_COMPILER = """#!/bin/sh
echo "$(basename $0) $*" >> "$LOG"
while [ $# -gt 0 ]; do [ "$1" = -o ] && : > "$2"; shift; done
"""


@pytest.fixture
def tree(tmp_path):
    """A copy of the sources with compilers that only note what they are asked for: tree(torch version or None) builds
    and returns the commands."""
    import shutil
    pkg = tmp_path / "pkg"
    shutil.copytree(os.path.join(ROOT, "paper_2407_04221_gb300", "csrc"), pkg / "csrc")
    shutil.copy(os.path.join(ROOT, "paper_2407_04221_gb300", "build.py"), pkg / "build.py")
    shutil.copytree(os.path.join(ROOT, "include"), tmp_path / "include")
    tools = tmp_path / "cuda" / "bin"
    tools.mkdir(parents=True)
    for name in ("nvcc", "g++"):
        (tools / name).write_text(FAKE_COMPILER)
        (tools / name).chmod(0o755)
    log = tmp_path / "log"

    def build(version):
        log.write_text("")
        fake = tmp_path / "site" / "torch"
        shutil.rmtree(fake, ignore_errors=True)
        fake.mkdir(parents=True)
        (fake / "__init__.py").write_text("raise ImportError('none')" if version is None else
                                          f"__version__ = {version!r}\nclass _C:\n    _GLIBCXX_USE_CXX11_ABI = True\n")
        env = dict(os.environ, CUDA_HOME=str(tmp_path / "cuda"), LOG=str(log), PYTHONPATH=str(tmp_path / "site"),
                   PATH=f"{tools}:{os.environ['PATH']}", PYTHONDONTWRITEBYTECODE="1")
        subprocess.run([sys.executable, "-c", "import build; build.build()"], cwd=pkg, env=env, check=True, timeout=120)
        return [line.split()[0] for line in log.read_text().splitlines()], (pkg / "_policy.so").exists()

    build.library = pkg / "libautoverse.so"
    return build


def test_the_library_is_built_without_torch(tree):
    commands, bound = tree(None)
    assert tree.library.exists() and set(commands) == {"nvcc"} and not bound
    assert tree(None) == ([], False)
    commands, bound = tree("1.0")  # torch came later: the binding alone
    assert commands == ["g++", "g++"] and bound


def test_the_binding_is_built_for_the_torch_that_is_there(tree):
    commands, bound = tree("1.0")
    assert "nvcc" in commands and "g++" in commands and bound
    assert tree("1.0") == ([], True)
    assert tree("1.1") == (["g++", "g++"], True)
    assert tree("1.1") == ([], True)


def test_statistics_off_their_alignment_are_refused():
    """Like every other pointer of the operators: an address that is never read."""
    import paper_2407_04221_gb300 as av
    L, P = av.load(), 0x10000
    ok = [4, 64, 1, 0, 1e-5, P, 64, P, P, P, 64, P, P, 0]
    for k in (11, 12):  # mean, rstd
        for bad in (P + 1, P + 2):
            assert L.av_layer_norm(*ok[:k], bad, *ok[k + 1:]) == -1, k
    ok = [4, 64, 1, 0, P, 64, P, 64, P, P, P, P, 64, P, P, P, 1 << 40, 0]
    for k in (9, 10):
        for bad in (P + 1, P + 2):
            assert L.av_layer_norm_grad(*ok[:k], bad, *ok[k + 1:]) == -1, k
