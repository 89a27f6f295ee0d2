"""Waits of the head's gradient that do not end, at stages that are known to be reached: the first and the last of G and of
the products, and one between (tests/late_counts.cu)."""
from __future__ import annotations

import ctypes
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")

from tests import test_gpu_policy_head as head  # noqa: E402
from tests.policy_ref import BF16, F16  # noqa: E402
from tests.test_gpu_policy_late import some_nan  # noqa: E402

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def pol():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2407_04221_gb300 import policy
    policy._load()
    return policy


@pytest.fixture(scope="module")
def late(pol, tmp_path_factory):
    import paper_2407_04221_gb300 as av
    from paper_2407_04221_gb300 import build
    lib = tmp_path_factory.mktemp("late") / "head_counts.so"
    subprocess.check_call([build.nvcc(), "-shared", "-O3", "-std=c++17", "-Xcompiler", "-fPIC", *build.ARCH, "-cudart", "shared",
                           "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, '-DAV_SOURCE="k_head.cu"',
                           os.path.join(HERE, "late_counts.cu"), "-o", str(lib), "-L", build.PKG, "-l:libautoverse.so",
                           "-Xlinker", "-rpath", "-Xlinker", build.PKG])
    L = ctypes.CDLL(str(lib))
    for name in av.EXPORTS:
        if hasattr(L, name):
            getattr(L, name).argtypes = getattr(av.load(), name).argtypes
    return L


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,D,V", [(5, 136, 500), (300, 136, 700), (3000, 264, 9000), (40, 1032, 300), (2000, 64, 3000)])
def test_head_gradient(pol, late, rows, D, V, dtype):
    """One piece of the words.  A block announces the blocks of terms of its tiles of G, then those of the products; a whole
    call counts them first.  A stage that comes short is one that the call waits for, so something is NaN: of G's both dx
    and dw, of the products' the one that the stage belongs to."""
    x, w, tok, dl = head.make(rows, D, V, dtype, rows)
    kind, st = {BF16: 1, F16: 2}[dtype], torch.cuda.current_stream().cuda_stream
    right = pol.head_log_probs(x, w, tok)
    grads = pol.head_log_probs_grad(dl, x, w, tok, right)
    need, calls = (ctypes.c_int64(), ctypes.c_int64()), ctypes.c_int()
    assert late.av_head_log_probs_work(rows, D, V, *(ctypes.byref(n) for n in need)) == 0
    work = torch.empty(need[1].value, dtype=torch.uint8, device="cuda")

    def run(nth):
        dx, dw = (torch.zeros_like(t) for t in grads)
        assert late.set_late(0, nth) == 0
        assert late.av_head_log_probs_grad(rows, D, V, kind, dl.data_ptr(), x.data_ptr(), D, w.data_ptr(), tok.data_ptr(), 8,
                                           right["peak"].data_ptr(), right["logz"].data_ptr(), dx.data_ptr(), D, dw.data_ptr(),
                                           work.data_ptr(), need[1].value, st) == 0
        torch.cuda.synchronize()
        assert late.late_count(ctypes.byref(calls)) == 0
        return dx, dw

    assert all(torch.equal(p, q) for p, q in zip(run(1 << 30), grads))
    everything, tiles, pairs = calls.value, -(-int((tok >= 0).sum()) // 256) * -(-V // 256), 76
    of_g = -(-tiles // pairs) * -(-D // 64)  # the first pair's share
    assert 0 < of_g < everything
    for nth in (0, of_g - 1, of_g, (of_g + everything) // 2, everything - 1):
        dx, dw = run(nth)
        assert calls.value > nth
        some_nan(dx, grads[0], 0, 1.0)
        some_nan(dw, grads[1], 0, 1.0)
        nan = torch.isnan(dx).any(), torch.isnan(dw).any()
        assert all(nan) if nth < of_g else any(nan), nth
