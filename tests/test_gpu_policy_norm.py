"""Layer norm and its gradient against the definition in 64 bits (tests/policy_ref.py)."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from tests import policy_ref as ref  # noqa: E402
from tests.policy_ref import BF16, E, F16, F32, close, d  # noqa: E402

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def pol():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2407_04221_gb300 import policy
    return policy


def make(rows, n, dtype, ptype, seed, loc=0.5):
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, n, generator=gen) * 2 + loc * torch.randn(rows, 1, generator=gen)).to(dtype)
    dy = torch.randn(rows, n, generator=gen).to(dtype)
    w = (1 + 0.3 * torch.randn(n, generator=gen)).to(ptype)
    b = (0.3 * torch.randn(n, generator=gen)).to(ptype)
    return x.cuda(), dy.cuda(), w.cuda(), b.cuda()


def check(pol, x, dy, w, b, what):
    """Bounds: a sum of n values taken 32 or more at a time is off by at most g = n / 32 + 16 roundings of the sum of
    magnitudes.  The mean is then off by e g mean|x|, the centred value by that and its own rounding, the variance
    relatively by (g + 8) e (its error in the mean is of second order), so xh by e (g + 8) |xh| + e (g + 2) mag, with
    mag = (mean|x| + |x|) rstd."""
    n = x.shape[-1]
    xd, dyd, wd, bd = (t.requires_grad_(t is not None) if t is not None else None for t in map(d, (x, dy, w, b)))
    y = ref.layer_norm(xd, wd, bd, EPS)
    got, mean, rstd = pol.layer_norm(x, w, b, eps=EPS)
    g = n / 32 + 16
    with torch.no_grad():
        m = xd.mean(-1, keepdim=True)
        r = 1 / ((xd - m).square().mean(-1, keepdim=True) + EPS).sqrt()
        xh = (xd - m) * r
        mag = (xd.abs().mean(-1, keepdim=True) + xd.abs()) * r
        near = (g + 8) * xh.abs() + (g + 2) * mag  # xh's error in units of e
        one = torch.ones(n, dtype=torch.float64)
        wa = one if wd is None else wd.abs()
        ba = 0 * one if bd is None else bd.abs()
    close(got, y, wa * near + 4 * (y.detach().abs() + ba), what + " y")
    close(mean, m[..., 0], (g + 2) * xd.detach().abs().mean(-1), what + " mean")
    close(rstd, r[..., 0], (g + 8 + (near.max(-1).values * 2)) * r[..., 0], what + " rstd")
    if dy is None:
        return
    grads = torch.autograd.grad((y * dyd).sum(), [t for t in (xd, wd, bd) if t is not None])
    dx, dw, db = pol.layer_norm_grad(dy, x, w, mean, rstd)
    with torch.no_grad():
        up = dyd.abs() * wa
        s1, s2 = up.mean(-1, keepdim=True), (up * xh.abs()).mean(-1, keepdim=True)
        s3 = (up * near).mean(-1, keepdim=True)
        scale = r * ((g + 12) * (up + s1 + xh.abs() * s2) + near * s2 + xh.abs() * s3)
        rows = xd.reshape(-1, n).shape[0]
        gr = rows / 8 + 64  # a column's sum, eight or more partial sums
        dscale = (dyd.abs() * near + gr * dyd.abs() * xh.abs()).reshape(-1, n).sum(0)
        bscale = gr * dyd.abs().reshape(-1, n).sum(0)
    close(dx, grads[0], scale, what + " dx")
    want_dw = grads[1] if wd is not None else (dyd * xh).reshape(-1, n).sum(0)
    close(dw, want_dw, dscale, what + " dw")
    close(db, grads[-1] if bd is not None else dyd.detach().reshape(-1, n).sum(0), bscale, what + " db")


@pytest.mark.parametrize("dtype,ptype", [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F16), (F16, F32)])
@pytest.mark.parametrize("rows,n", [(1, 1), (3, 5), (7, 32), (5, 33), (300, 64), (1000, 96), (64, 256), (9, 1000),
                                    (33, 1024), (257, 2048), (3, 4097), (5, 8192), (2, 16384), (3, 20011)])
def test_norm(pol, rows, n, dtype, ptype):
    check(pol, *make(rows, n, dtype, ptype, rows * n), f"{rows}x{n} {dtype} {ptype}")


@pytest.mark.parametrize("n", [24, 1000, 1024, 3001])
def test_many_rows(pol, n):
    """More rows than blocks hold at once."""
    rows = 20000 if n < 2000 else 6007
    check(pol, *make(rows, n, BF16, F32, n), f"{rows}x{n}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [8, 40, 1024, 5000])
def test_strides_and_starts(pol, dtype, n):
    """Rows of a wider array from an odd start, three axes, one row for all."""
    x, dy, w, b = make(24, n + 9, dtype, F32, n)
    w, b = w[:n].contiguous(), b[:n].contiguous()
    check(pol, x[:, 1:n + 1], dy[:, 8:n + 8], w, b, "offset")
    check(pol, x[:, 8:n + 8].unflatten(0, (4, 6)), dy[:, :n].unflatten(0, (4, 6)), w, b, "three axes")
    check(pol, x[:1, :n].expand(24, n), dy[:, :n], w, b, "one row")
    check(pol, x[::2, :n], dy[::2, :n], w, b, "every second row")


def test_without_parameters(pol):
    x, dy, w, b = make(50, 200, BF16, F32, 3)
    check(pol, x, dy, None, None, "plain")
    check(pol, x, dy, w, None, "weight")


@pytest.mark.parametrize("n", [16, 700, 9000])
def test_constant_and_shifted_rows(pol, n):
    """A row of one value has no spread: y is the bias; far from 0 the spread must not drown in the mean."""
    x, dy, w, b = make(40, n, F32, F32, n, loc=3000.0)
    x[7] = 2.5
    check(pol, x, dy, w, b, "shifted")
    y, _, rstd = pol.layer_norm(x, w, b, eps=EPS)
    assert torch.equal(y[7], b) and abs(float(rstd[7]) - EPS**-0.5) < 1e-4 * EPS**-0.5


def test_bad_values_stay_in_their_row(pol):
    x, dy, w, b = make(64, 520, F32, F32, 1)
    good = pol.layer_norm(x, w, b)
    x[3, 17], x[9, 0] = float("nan"), float("inf")
    y, mean, rstd = pol.layer_norm(x, w, b)
    keep = [r for r in range(64) if r not in (3, 9)]
    assert torch.equal(y[keep], good[0][keep]) and torch.isnan(y[[3, 9]]).all()


@pytest.mark.parametrize("rows,n", [(0, 64), (0, 5000)])
def test_no_rows(pol, rows, n):
    x, dy, w, b = make(rows, n, BF16, F32, 1)
    y, mean, rstd = pol.layer_norm(x, w, b)
    dx, dw, db = pol.layer_norm_grad(dy, x, w, mean, rstd)
    assert y.shape == dx.shape == (0, n) and not dw.any() and not db.any()


@pytest.mark.parametrize("n", [12, 777])
def test_gradient_against_differences(pol, n):
    """Central differences of the kernel's own forward pass, in f32.  Along a unit direction the loss L = sum c y has
    a third derivative of order sqrt(rows n) rstd^2: with a step of 2^-5 the truncation is below 2^-10 of L's slope
    scale |c|, and rounding adds at most e |c| |y| 2^5 ~ 2^-12 sqrt(n rows); the bound is 1 % of |dx| plus that."""
    x, c, w, b = make(16, n, F32, F32, n)
    y, mean, rstd = pol.layer_norm(x, w, b)
    dx, dw, db = pol.layer_norm_grad(c, x, w, mean, rstd)
    gen = torch.Generator().manual_seed(n)
    h = 2.0**-5
    for k, (target, grad) in enumerate(((x, dx), (w, dw), (b, db))):
        v = torch.randn(target.shape, generator=gen)
        v = (v / v.norm()).cuda()
        args = [x, w, b]
        side = []
        for s in (h, -h):
            args[k] = target + s * v
            side.append(float((pol.layer_norm(*args)[0].double() * c.double()).sum()))
        slope, want = (side[0] - side[1]) / (2 * h), float((grad.double() * v.double()).sum())
        assert abs(slope - want) <= 0.01 * float(grad.double().norm()) + E / h * float((y * c).abs().double().sum())


def test_same_bits_again(pol):
    x, dy, w, b = make(5000, 1000, BF16, F32, 5)
    _, mean, rstd = pol.layer_norm(x, w, b)
    first = pol.layer_norm_grad(dy, x, w, mean, rstd)
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(first, pol.layer_norm_grad(dy, x, w, mean, rstd)))
