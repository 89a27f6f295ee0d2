"""A wait for a copy that does not end (tests/late_copies.cu): the call returns, and whatever the missing bytes would have
touched is NaN, so that nothing wrong passes for right."""
from __future__ import annotations

import ctypes
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

torch = pytest.importorskip("torch")

from tests import test_gpu_policy_ffn as ffn  # noqa: E402
from tests import test_gpu_policy_norm as norm  # noqa: E402
from tests import test_gpu_policy_scan as scan  # noqa: E402
from tests.policy_ref import BF16, F16, F32  # noqa: E402

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def late(tmp_path_factory):
    """The libraries with an operator's kernels compiled so, argument types as the package's, by their source."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2407_04221_gb300 as av
    from paper_2407_04221_gb300 import build, policy
    policy._load()
    ours, at = av.load(), tmp_path_factory.mktemp("late")

    def made(source):
        lib = at / (source + ".so")
        subprocess.check_call([build.nvcc(), "-shared", "-O3", "-std=c++17", "-Xcompiler", "-fPIC", *build.ARCH, "-cudart",
                               "shared", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC,
                               f'-DAV_SOURCE="{source}"', os.path.join(HERE, "late_copies.cu"), "-o", str(lib),
                               "-L", build.PKG, "-l:libautoverse.so", "-Xlinker", "-rpath", "-Xlinker", build.PKG])
        L = ctypes.CDLL(str(lib))
        for name in av.EXPORTS:
            if hasattr(L, name):
                getattr(L, name).argtypes = getattr(ours, name).argtypes
        return L

    sources = ("k_norm.cu", "k_scan.cu", "k_ffn.cu")
    with ThreadPoolExecutor(len(sources)) as pool:
        return dict(zip(sources, pool.map(made, sources)))


@pytest.fixture(scope="module")
def pol(late):
    from paper_2407_04221_gb300 import policy
    return policy


@pytest.fixture(scope="module")
def late_norm(late):
    return late["k_norm.cu"]


def right_or_nan(got, right):
    """Of rows of values: which are right throughout; the others are NaN throughout."""
    good, bad = (got == right).all(-1), torch.isnan(got).all(-1)
    assert (good | bad).all()
    return good


@pytest.mark.parametrize("n,dtype", [(1024, BF16), (1001, F32), (4805, F32)])
def test_layer_norm(pol, late_norm, n, dtype):
    rows = 6000
    x, dy, w, b = norm.make(rows, n, dtype, F32, n)
    kind, st = {F32: 0, BF16: 1}[dtype], torch.cuda.current_stream().cuda_stream
    right = pol.layer_norm(x, w, b)
    grads = pol.layer_norm_grad(dy, x, w, *right[1:])
    y, mean, rstd = (torch.zeros_like(t) for t in right)
    for nth in (0, 1):  # (a group takes two rows at least)
        assert late_norm.set_late(1, nth) == 0
        assert late_norm.av_layer_norm(rows, n, kind, 0, norm.EPS, x.data_ptr(), n, w.data_ptr(), b.data_ptr(),
                                       y.data_ptr(), n, mean.data_ptr(), rstd.data_ptr(), st) == 0
        torch.cuda.synchronize()
        good = right_or_nan(y, right[0])
        assert 0 < int((~good).sum()) < rows // 2
        for got, want in ((mean, right[1]), (rstd, right[2])):
            assert torch.equal(got[good], want[good]) and torch.isnan(got[~good]).all()
        dx, dw, db = (torch.zeros_like(t) for t in grads)
        need = ctypes.c_int64()
        assert late_norm.av_layer_norm_work(rows, n, ctypes.byref(need)) == 0
        work = torch.empty(need.value, dtype=torch.uint8, device="cuda")
        assert late_norm.set_late(1, nth) == 0
        assert late_norm.av_layer_norm_grad(rows, n, kind, 0, dy.data_ptr(), n, x.data_ptr(), n, w.data_ptr(),
                                            right[1].data_ptr(), right[2].data_ptr(), dx.data_ptr(), n, dw.data_ptr(),
                                            db.data_ptr(), work.data_ptr(), need.value, st) == 0
        torch.cuda.synchronize()
        assert 0 < int((~right_or_nan(dx, grads[0])).sum()) < rows // 2
        assert torch.isnan(dw).all() and torch.isnan(db).all()
    assert late_norm.set_late(-1, 0) == 0  # (no block's)
    assert late_norm.av_layer_norm(rows, n, kind, 0, norm.EPS, x.data_ptr(), n, w.data_ptr(), b.data_ptr(), y.data_ptr(), n,
                                   mean.data_ptr(), rstd.data_ptr(), st) == 0
    assert torch.equal(y, right[0])


def some_nan(got, right, least=1, most=0.5):
    """Values are right or NaN; how many are NaN is within least and a share of them."""
    bad = got != right
    assert torch.isnan(got[bad]).all() and least <= int(bad.sum()) <= most * bad.numel()


@pytest.fixture(scope="module")
def late_scan(late):
    return late["k_scan.cu"]


@pytest.mark.parametrize("T,B,D,dtype", [(700, 400, 64, BF16), (700, 400, 65, BF16), (700, 400, 66, BF16),
                                         (700, 400, 64, F32), (3001, 8, 64, BF16), (3001, 8, 65, F32)])
@pytest.mark.parametrize("resets", [0.0, 0.02])
def test_scan(pol, late_scan, T, B, D, dtype, resets):
    """By tensor copies and by rows, whole and in segments (the last two).  Begins of episodes do not end the NaN within
    a block, which knows nothing of the steps that it missed."""
    g, v, reset, h0, dh, dlast = scan.make(T, B, D, dtype, resets, T + D, shift=3.0)
    kind, st = {F32: 0, BF16: 1}[dtype], torch.cuda.current_stream().cuda_stream
    h, last, states = pol.scan(g, v, reset, h0, save=True)
    grads = pol.scan_grad(dh, g, v, reset, states, dlast=dlast)
    sizes = ctypes.c_int64(), ctypes.c_int64()
    assert late_scan.av_scan_sizes(T, B, D, kind, *(ctypes.byref(n) for n in sizes)) == 0
    work = torch.empty(max(16, sizes[1].value), dtype=torch.uint8, device="cuda")
    t, b = B * D, D
    args = [g.data_ptr(), t, b, v.data_ptr(), t, b, reset.data_ptr(), B, 1]
    for nth in (0, 1):
        got = [torch.zeros_like(x) for x in (h, last, states)]
        assert late_scan.set_late(1, nth) == 0
        assert late_scan.av_scan(T, B, D, kind, *args, h0.data_ptr(), got[0].data_ptr(), t, b, got[1].data_ptr(),
                                 got[2].data_ptr(), work.data_ptr(), sizes[1].value, st) == 0
        torch.cuda.synchronize()
        some_nan(got[0], h)
        some_nan(got[1], last, 0)
        some_nan(got[2], states, 0)
        got = [torch.zeros_like(x) for x in grads]
        assert late_scan.set_late(1, nth) == 0
        assert late_scan.av_scan_grad(T, B, D, kind, dh.data_ptr(), t, b, *args, states.data_ptr(), dlast.data_ptr(),
                                      got[0].data_ptr(), t, b, got[1].data_ptr(), t, b, got[2].data_ptr(), work.data_ptr(),
                                      sizes[1].value, st) == 0
        torch.cuda.synchronize()
        some_nan(got[0], grads[0])
        some_nan(got[1], grads[1])
        some_nan(got[2], grads[2], 0)


@pytest.fixture(scope="module")
def late_ffn(late):
    return late["k_ffn.cu"]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,D,H", [(300, 136, 264), (9000, 264, 520), (40, 2056, 72)])
def test_gated_ffn(pol, late_ffn, rows, D, H, dtype):
    """One tile a pair of blocks, several, and terms in parts.  The first pair's copies come short, those of its first
    CTA's first or a later stage: of h, of dg and du, of dx or of dw (by the count of stages before)."""
    x, w, dh = ffn.make(rows, D, H, dtype, rows)
    kind, st = {BF16: 1, F16: 2}[dtype], torch.cuda.current_stream().cuda_stream
    right, grads = pol.gated_ffn(x, w), pol.gated_ffn_grad(dh, x, w)
    need = ctypes.c_int64()
    assert late_ffn.av_gated_ffn_work(rows, D, H, ctypes.byref(need)) == 0
    work = torch.empty(need.value, dtype=torch.uint8, device="cuda")
    blocks = -(-D // 64)
    for nth in (0, blocks - 1, blocks + 1):
        h = torch.zeros_like(right)
        assert late_ffn.set_late(0, nth) == 0
        assert late_ffn.av_gated_ffn(rows, D, H, kind, 0, x.data_ptr(), D, w.data_ptr(), h.data_ptr(), H, st) == 0
        torch.cuda.synchronize()
        some_nan(h, right, 0 if nth > blocks else 1, 1.0)
    for nth in (0, blocks, blocks + 2, blocks + 40, blocks + 90):
        dx, dw = (torch.zeros_like(t) for t in grads)
        assert late_ffn.set_late(0, nth) == 0
        assert late_ffn.av_gated_ffn_grad(rows, D, H, kind, 0, dh.data_ptr(), H, x.data_ptr(), D, w.data_ptr(),
                                          dx.data_ptr(), D, dw.data_ptr(), work.data_ptr(), need.value, st) == 0
        torch.cuda.synchronize()
        some_nan(dx, grads[0], 0, 1.0)
        some_nan(dw, grads[1], 0, 1.0)
        assert nth > 0 or (torch.isnan(dx).any() and torch.isnan(dw).any())
