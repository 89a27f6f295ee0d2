"""What the policy operators refuse, before any GPU work (no GPU needed)."""
from __future__ import annotations

import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2407_04221_gb300 import build
    build.build()
    import paper_2407_04221_gb300 as av
    return av.load()


P = 0x10000  # an address that is never read: every call here is refused, or has nothing to do


def test_layer_norm(lib):
    ok = [4, 64, 1, 0, 1e-5, P, 64, P, P, P, 64, P, P, 0]
    for k, bad in ((0, -1), (0, 1 << 60), (1, 0), (1, -5), (2, 3), (2, -1), (3, 7), (4, -1.0), (4, float("nan")), (5, None),
                   (5, P + 1), (6, -64), (7, P + 2), (8, P + 1), (9, None), (9, P + 1), (10, 63), (10, 0), (11, None),
                   (12, None)):
        a = list(ok)
        a[k] = bad
        assert lib.av_layer_norm(*a) == -1, (k, bad)
    assert lib.av_layer_norm(0, 64, 1, 0, 1e-5, None, 64, None, None, None, 64, None, None, 0) == 0
    need = ctypes.c_int64(-1)
    assert lib.av_layer_norm_work(4, 64, ctypes.byref(need)) == 0 and need.value >= 0
    assert lib.av_layer_norm_work(4, 64, None) == lib.av_layer_norm_work(4, 0, ctypes.byref(need)) == -1
    ok = [4, 64, 1, 0, P, 64, P, 64, P, P, P, P, 64, P, P, P, 1 << 40, 0]
    for k, bad in ((0, -1), (1, 0), (2, 3), (3, 3), (4, None), (5, -1), (6, None), (6, P + 1), (8, P + 1), (9, None),
                   (10, None), (11, None), (12, 60), (13, P + 2), (14, P + 1)):
        a = list(ok)
        a[k] = bad
        assert lib.av_layer_norm_grad(*a) == -1, (k, bad)


def test_scan(lib):
    ok = [5, 3, 16, 1, P, 48, 16, P, 48, 16, P, 3, 1, P, P, 48, 16, P, P, P, 1 << 40, 0]
    for k, bad in ((0, -1), (1, -1), (2, -1), (0, 1 << 47), (3, 3), (4, None), (4, P + 1), (5, -48), (6, -1), (7, None),
                   (8, -1), (11, -1), (13, P + 2), (14, None), (14, P + 1), (15, 16), (15, 0), (16, 8), (16, 0),
                   (17, P + 1), (18, P + 3)):
        a = list(ok)
        a[k] = bad
        assert lib.av_scan(*a) == -1, (k, bad)
    assert lib.av_scan(5, 0, 16, 1, *[None, 0, 0] * 3, None, None, 0, 0, None, None, None, 0, 0) == 0
    s, w = ctypes.c_int64(), ctypes.c_int64()
    assert lib.av_scan_sizes(5, 3, 16, 1, ctypes.byref(s), ctypes.byref(w)) == 0 and s.value >= 48
    assert lib.av_scan_sizes(5, 3, 16, 9, ctypes.byref(s), ctypes.byref(w)) == -1
    assert lib.av_scan_sizes(5, 3, 16, 1, None, ctypes.byref(w)) == -1
    ok = [5, 3, 16, 1, P, 48, 16, P, 48, 16, P, 48, 16, P, 3, 1, P, P, P, 48, 16, P, 48, 16, P, P, 1 << 40, 0]
    for k, bad in ((0, -1), (3, 4), (4, None), (5, -1), (7, None), (10, P + 1), (16, None), (17, P + 1), (18, None),
                   (19, 16), (20, 15), (21, None), (22, 0), (24, P + 2)):
        a = list(ok)
        a[k] = bad
        assert lib.av_scan_grad(*a) == -1, (k, bad)


def test_scan_workspace(lib):
    """A long sequence needs its workspace."""
    s, w = ctypes.c_int64(), ctypes.c_int64()
    assert lib.av_scan_sizes(100000, 1, 16, 0, ctypes.byref(s), ctypes.byref(w)) == 0
    if w.value:
        ok = [100000, 1, 16, 0, P, 16, 16, P, 16, 16, None, 0, 0, P, P, 16, 16, P, P, P, w.value, 0]
        for k, bad in ((19, None), (19, P + 8), (20, w.value - 1), (20, 0)):
            a = list(ok)
            a[k] = bad
            assert lib.av_scan(*a) == -1, (k, bad)


def test_log_probs(lib):
    ok = [4, 100, 1, P, 100, P, 8, P, 100, 3, P, P, P, P, P, P, 0]
    for k, bad in ((0, -1), (0, 1 << 60), (1, 0), (2, 5), (3, None), (3, P + 1), (4, -1), (5, None), (5, P + 4), (6, 2),
                   (6, 0), (8, -1), (9, -1), (9, 33), (10, None), (10, P + 2), (14, None), (15, None)):
        a = list(ok)
        a[k] = bad
        assert lib.av_log_probs(*a) == -1, (k, bad)
    assert lib.av_log_probs(4, 2, 1, P, 2, P, 8, None, 0, 3, P, P, P, P, P, P, 0) == -1  # more than there are
    assert lib.av_log_probs(0, 2, 1, None, 2, None, 8, None, 0, 1, None, None, None, None, None, None, 0) == 0
    ok = [4, 100, 1, P, 100, P, 8, P, 100, P, P, P, P, P, P, 100, 0]
    for k, bad in ((0, -1), (1, -1), (2, 5), (3, None), (5, None), (6, 3), (11, None), (12, None), (13, None), (14, None),
                   (14, P + 1), (15, 99)):
        a = list(ok)
        a[k] = bad
        assert lib.av_log_probs_grad(*a) == -1, (k, bad)


def test_gated_ffn(lib):
    ok = [4, 64, 72, 1, 0, P, 64, P, P, 72, 0]
    for k, bad in ((0, -1), (0, 1 << 40), (1, 0), (1, 60), (2, 4), (2, 71), (3, 0), (3, 3), (4, 2), (5, None), (5, P + 8),
                   (6, 56), (6, 65), (7, None), (7, P + 4), (8, None), (8, P + 2), (9, 64), (9, 73)):
        a = list(ok)
        a[k] = bad
        assert lib.av_gated_ffn(*a) == -1, (k, bad)
    assert lib.av_gated_ffn(0, 64, 72, 1, 0, None, 64, None, None, 72, 0) == 0
    need = ctypes.c_int64()
    assert lib.av_gated_ffn_work(4, 64, 72, ctypes.byref(need)) == 0 and need.value > 0
    assert lib.av_gated_ffn_work(4, 64, 70, ctypes.byref(need)) == -1
    ok = [4, 64, 72, 1, 0, P, 72, P, 64, P, P, 64, P, P, need.value, 0]
    for k, bad in ((0, -1), (1, 12), (3, 0), (4, -1), (5, None), (6, 64), (7, P + 8), (8, 60), (9, None), (10, None),
                   (11, 8), (12, P + 8), (13, None), (13, P + 8), (14, need.value - 1)):
        a = list(ok)
        a[k] = bad
        assert lib.av_gated_ffn_grad(*a) == -1, (k, bad)


def test_binding_refuses_what_it_cannot_pass():
    torch = pytest.importorskip("torch")
    from paper_2407_04221_gb300 import policy as pol
    x = torch.zeros(4, 64)
    for call in (lambda: pol.layer_norm(x), lambda: pol.scan(x[None], x[None]), lambda: pol.gated_ffn(x, x),
                 lambda: pol.log_probs(x, torch.zeros(4, dtype=torch.int64)), lambda: pol.layer_norm(None),
                 lambda: pol.layer_norm(x, stream=5)):
        with pytest.raises(ValueError):
            call()
