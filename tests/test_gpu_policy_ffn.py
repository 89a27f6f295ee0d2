"""The gated feed-forward and its gradient against the definition in 64 bits (tests/policy_ref.py)."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from tests import policy_ref as ref  # noqa: E402
from tests.policy_ref import BF16, E, F16, ROUNDOFF, close, d  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pol():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2407_04221_gb300 import policy
    return policy


def make(rows, D, H, dtype, seed, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, D, generator=gen).to(dtype).cuda()
    w = (scale * torch.randn(2, H, D, generator=gen) / D**0.5).to(dtype).cuda()
    dh = torch.randn(rows, H, generator=gen).to(dtype).cuda()
    return x, w, dh


def check(pol, x, w, dh, act, what):
    """Bounds: a product's sum of D terms in 32 bits, truncated or rounded term by term, is off by at most
    2 e D sum |x| |w|; the activation's slope is below 1.13 and it is good to (|g| + 16) e relatively.  The
    projections' gradients are rounded to the type, u, before the next products."""
    u, D, H = ROUNDOFF[x.dtype], x.shape[-1], w.shape[1]
    xd, wd = d(x).reshape(-1, D).requires_grad_(), d(w).requires_grad_()
    rows = xd.shape[0]
    h = ref.gated_ffn(xd, wd, act)
    with torch.no_grad():
        g, up = xd @ wd[0].t(), xd @ wd[1].t()
        ge, ue = (2 * D * (xd.abs() @ wd[k].abs().t()) for k in (0, 1))
        f = ref.activate(g, act)
        fe = 1.13 * ge + (g.abs() + 16) * (f.abs() + 1e-3)
    close(pol.gated_ffn(x, w, act=act).reshape(-1, H), h, fe * up.abs() + f.abs() * ue + 4 * (f * up).abs(), what + " h")
    dhd = d(dh).reshape(-1, H)
    want = torch.autograd.grad((h * dhd).sum(), [xd, wd])
    dx, dw = pol.gated_ffn_grad(dh, x, w, act=act)
    with torch.no_grad():
        gg = g.clone().requires_grad_()
    with torch.enable_grad():
        (slope,) = torch.autograd.grad(ref.activate(gg, act).sum(), gg)
    a = dhd.abs()
    # the gradients of the projections, their 32-bit error in units of e, and their rounding
    dg, du = a * up.abs() * slope.abs(), a * f.abs()
    # (the slope's slope is below 0.8 for either activation)
    dge, due = a * (ue * 1.13 + up.abs() * (0.8 * ge + g.abs() + 24)), a * fe
    er = [1.01 * u * dg + E * dge, 1.01 * u * du + E * due]
    wa, xa = d(w).abs(), xd.detach().abs()
    close(dx.reshape(-1, D), want[0], 4 * H * (dg @ wa[0] + du @ wa[1]), what + " dx", er[0] @ wa[0] + er[1] @ wa[1])
    close(dw, want[1], 2 * rows * torch.stack((dg.t() @ xa, du.t() @ xa)), what + " dw",
          torch.stack((er[0].t() @ xa, er[1].t() @ xa)))


@pytest.mark.parametrize("dtype,act", [(BF16, "silu"), (F16, "gelu")])
@pytest.mark.parametrize("rows,D,H", [(1, 8, 8), (1, 1024, 264), (2, 64, 136), (5, 520, 72), (8, 128, 128), (9, 72, 64),
                                      (16, 256, 512), (17, 64, 64), (64, 128, 256), (100, 40, 24), (127, 64, 128),
                                      (128, 64, 128), (129, 136, 136), (257, 264, 520), (300, 512, 1368),
                                      (1000, 200, 88), (2049, 64, 72)])
def test_gated_ffn(pol, rows, D, H, dtype, act):
    check(pol, *make(rows, D, H, dtype, rows + D + H), act, f"{rows} {D} {H} {dtype} {act}")


@pytest.mark.parametrize("dtype,act", [(BF16, "gelu"), (F16, "silu")])
@pytest.mark.parametrize("rows", [3, 40, 200, 700])
def test_types_and_activations(pol, rows, dtype, act):
    check(pol, *make(rows, 192, 328, dtype, rows), act, f"{rows} {dtype} {act}")


@pytest.mark.parametrize("rows", [6, 60, 300])
def test_strides(pol, rows):
    """Rows of wider arrays, from starts of whole eights; three axes."""
    x, w, dh = make(rows, 64 + 24, 136 + 8, BF16, rows)
    w = w[:, :136, :64].contiguous()
    check(pol, x[:, 8:72], w, dh[:, 8:144], "silu", "wide")
    check(pol, x[:, :64].unflatten(0, (2, -1)), w, dh[:, :136].unflatten(0, (2, -1)), "silu", "axes")


def test_large_gates(pol):
    """Gates far out, where the activations are 0 or the gate itself."""
    check(pol, *make(70, 64, 64, BF16, 1, scale=30.0), "silu", "silu")
    check(pol, *make(70, 64, 64, BF16, 2, scale=30.0), "gelu", "gelu")


@pytest.mark.parametrize("rows", [3, 150])
def test_bad_values_stay_in_their_row(pol, rows):
    x, w, dh = make(rows, 72, 88, BF16, rows)
    good = pol.gated_ffn(x, w), pol.gated_ffn_grad(dh, x, w)[0]
    x[1, 5] = float("nan")
    keep = [r for r in range(rows) if r != 1]
    h = pol.gated_ffn(x, w)
    assert torch.equal(h[keep], good[0][keep]) and torch.isnan(h[1]).all()
    dx, dw = pol.gated_ffn_grad(dh, x, w)
    assert torch.equal(dx[keep], good[1][keep]) and torch.isnan(dx[1]).all() and torch.isnan(dw).all()


def test_no_rows(pol):
    x, w, dh = make(0, 64, 72, BF16, 1)
    assert pol.gated_ffn(x, w).shape == (0, 72)
    dx, dw = pol.gated_ffn_grad(dh, x, w)
    assert dx.shape == (0, 64) and not dw.any()


@pytest.mark.parametrize("rows", [5, 200])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradient_against_differences(pol, rows, act):
    """Central differences of the kernel's own forward pass, f16, along directions of the arrays' own grid (so that
    both sides are representable): h's rounding, u, limits them to u |h dh| / step per output, at random signs its
    root sum of squares (4 times that is allowed), and truncation is of order step^2 of the slope, 2 % here."""
    x, w, dh = make(rows, 64, 72, F16, rows)
    dx, dw = pol.gated_ffn_grad(dh, x, w, act=act)
    gen = torch.Generator().manual_seed(rows)
    for k, (at, grad) in enumerate(((x, dx), (w, dw))):
        step = (2.0**-4 if k == 0 else 2.0**-7) * torch.randint(-1, 2, at.shape, generator=gen).to(at.dtype).cuda()
        hi, lo = at + step, at - step
        move = hi.double() - lo.double()
        hs = [pol.gated_ffn(*((y, w) if k == 0 else (x, y)), act=act).double() for y in (hi, lo)]
        got = float(((hs[0] - hs[1]) * dh.double()).sum())
        want = float((grad.double() * move).sum())
        noise = float((hs[0] * dh.double()).square().sum().sqrt()) * ROUNDOFF[F16] * 2**0.5
        assert abs(got - want) <= 4 * noise + 0.02 * float((grad.double() * move).square().sum().sqrt()) + 0.02 * abs(want)


def test_same_bits_again(pol):
    x, w, dh = make(3001, 264, 520, BF16, 5)
    first = (pol.gated_ffn(x, w), *pol.gated_ffn_grad(dh, x, w))
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(first, (pol.gated_ffn(x, w), *pol.gated_ffn_grad(dh, x, w))))
