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
