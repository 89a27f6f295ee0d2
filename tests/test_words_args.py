"""What the operators over cell words refuse, before any GPU work (no GPU needed)."""
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


def refused(call, ok, cases):
    for k, bad in cases:
        a = list(ok)
        a[k] = bad
        assert call(*a) == -1, (k, bad)


def test_embed(lib):
    ok = [5, 100, 24, 0, 1, 1.0, P, 8, P, P, 24, 0]
    refused(lib.av_embed, ok, ((0, -1), (0, 1 << 30), (1, 0), (1, 1 << 30), (2, 0), (2, 1 << 20), (3, 3), (4, -1), (6, None),
                               (6, P + 4), (7, 3), (8, None), (8, P + 2), (9, None), (9, P + 1), (10, 23), (10, 0), (10, -24)))
    assert lib.av_embed(0, 100, 24, 0, 1, 1.0, None, 8, None, None, 24, 0) == 0
    need = ctypes.c_int64(-1)
    assert lib.av_embed_work(5, 100, 24, ctypes.byref(need)) == 0 and need.value > 0
    for bad in ((5, 100, 0), (-1, 100, 24), (5, 0, 24), (5, 1 << 30, 24)):
        assert lib.av_embed_work(*bad, ctypes.byref(need)) == -1
    assert lib.av_embed_work(5, 100, 24, None) == -1
    assert lib.av_embed_work(5, 100, 24, ctypes.byref(need)) == 0
    ok = [5, 100, 24, 1, 0, 1.0, P, 4, P, 24, P, P, need.value, 0]
    refused(lib.av_embed_grad, ok, ((0, -1), (1, 0), (2, -3), (3, 5), (4, 3), (6, None), (6, P + 2), (7, 3), (8, None), (8, P + 1),
                                    (9, -1), (10, None), (10, P + 2), (11, None), (11, P + 8), (12, need.value - 1)))


def test_head(lib):
    fwd, grad = ctypes.c_int64(-1), ctypes.c_int64(-1)
    work = lambda *a: lib.av_head_log_probs_work(*a, ctypes.byref(fwd), ctypes.byref(grad))  # noqa: E731
    assert work(40, 64, 100) == 0 and fwd.value > 0 and grad.value > 0
    for bad in ((-1, 64, 100), (40, 60, 100), (40, 0, 100), (40, 64, 0), (1 << 30, 64, 100), (40, 64, 1 << 30), (1 << 29, 8, 1 << 29)):
        assert work(*bad) == -1, bad
    assert lib.av_head_log_probs_work(40, 64, 100, None, ctypes.byref(grad)) == -1
    assert lib.av_head_log_probs_work(40, 64, 100, ctypes.byref(fwd), None) == -1
    assert work(40, 64, 100) == 0
    ok = [40, 64, 100, 1, P, 64, P, P, 8, P, P, P, P, fwd.value, 0]
    refused(lib.av_head_log_probs, ok, ((0, -1), (1, 60), (2, 0), (3, 0), (3, 3), (4, None), (4, P + 8), (5, 56), (5, 68), (6, None),
                                        (6, P + 2), (7, None), (7, P + 4), (8, 16), (9, None), (9, P + 2), (10, P + 1), (11, P + 3),
                                        (12, None), (12, P + 16), (13, fwd.value - 1)))
    assert lib.av_head_log_probs(0, 64, 100, 1, None, 64, None, None, 8, None, None, None, None, 0, 0) == 0
    ok = [40, 64, 100, 2, P, P, 64, P, P, 4, P, P, P, 64, P, P, grad.value, 0]
    refused(lib.av_head_log_probs_grad, ok, ((0, -1), (1, 12), (2, -1), (3, 0), (4, None), (4, P + 2), (5, None), (5, P + 8), (6, 60),
                                             (7, None), (8, None), (8, P + 2), (9, 5), (10, None), (10, P + 1), (11, None),
                                             (12, None), (12, P + 8), (13, 8), (13, 65), (14, None), (14, P + 8), (15, None),
                                             (15, P + 128), (16, grad.value - 1)))


def test_distill(lib):
    ok = [4, 100, 1, P, 100, P, 0, P, 4, 8, 1.0, P, 100, P, P, P, 0]
    bad = [(0, -1), (0, 1 << 31), (1, 0), (2, 3), (3, None), (3, P + 1), (4, -1), (5, None), (5, P + 2), (6, 4), (7, None),
           (7, P + 2), (8, 1), (9, 0), (9, 101), (9, 257), (10, 0.0), (10, -1.0), (10, float("nan")), (10, float("inf")),
           (10, 1e-39), (12, -1)]
    refused(lib.av_distill, ok, bad + [(13, None), (13, P + 1), (14, P + 2), (15, P + 2)])
    assert lib.av_distill(4, 1000, 1, P, 1000, P, 0, P, 4, 257, 1.0, None, 0, P, P, P, 0) == -1
    assert lib.av_distill(0, 100, 1, None, 100, None, 0, None, 4, 8, 1.0, None, 0, None, None, None, 0) == 0
    ok = ok[:13] + [P, P, P, P, 100, 0]
    refused(lib.av_distill_grad, ok, bad + [(13, None), (13, P + 1), (14, None), (15, None), (15, P + 2), (16, None), (16, P + 1),
                                            (17, 99)])


def test_binding_refuses_what_it_cannot_pass():
    torch = pytest.importorskip("torch")
    from paper_2407_04221_gb300 import policy as pol
    x, tok = torch.zeros(4, 64), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: pol.embed(tok, x), lambda: pol.embed_grad(x, tok, 9), lambda: pol.head_log_probs(x, x, tok),
                 lambda: pol.head_log_probs_grad(x[:, 0], x, x, tok, dict(peak=x[:, 0], logz=x[:, 0])),
                 lambda: pol.distill(x, x[:, :2], tok[:, None]), lambda: pol.embed(None, None),
                 lambda: pol.distill_grad(x[:, 0], x, x, tok, dict(peak=None, logz=None)), lambda: pol.embed(tok, x, stream=5)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("temperature", [1.5e-39, 3.4e-39, 4.9e-39])
def test_distill_temperatures_too_low(lib, temperature):
    """1 / temperature times log2(e) has to be finite: else the peak would be 0 times infinity."""
    forward = [4, 100, 1, P, 100, P, 0, P, 4, 8, temperature, None, 0, P, P, P, 0]
    assert lib.av_distill(*forward) == -1
    assert lib.av_distill_grad(*forward[:13], P, P, P, P, 100, 0) == -1
    ok = [0, 100, 1, None, 100, None, 0, None, 4, 8, 2.0**-126, None, 0, None, None, None, 0]
    assert lib.av_distill(*ok) == 0
