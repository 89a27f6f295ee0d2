"""What the policy operators' gradients may lose: no more than rounding the result once, whatever the sizes, and of
32-bit logits no more than the formula's own operations."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from tests import test_gpu_policy_ffn as ffn  # noqa: E402
from tests.policy_ref import BF16, F16, d, gated_ffn  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pol():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2407_04221_gb300 import policy
    return policy


# ------------------------------------------------------------ gated feed-forward

def rounded_once(pol, x, w, dh, act, what):
    """The root mean square of the gradients' errors against that of rounding the exact gradients, which is 0.3 to 0.45
    u of theirs (or a fixed step, for subnormal ones).  What comes before: the projections' gradients as two values
    each are off by 2 u^2; a sum of K terms, sixteen at a time, by a truncation of 2^-23 of its partial sum at every
    addition, K / 16 of them, half of it on average, and the partial sums of terms of random sign grow with the square
    root, so that the mean one is below the result: K 2^-28, of K <= 2^13 terms 2^-15, or 0.2 of f16's 0.3 x 2^-11.  In
    quadrature that is 1.02; 1.05 is allowed."""
    xd, wd = d(x).requires_grad_(), d(w).requires_grad_()
    want = torch.autograd.grad((gated_ffn(xd, wd, act) * d(dh)).sum(), [xd, wd])
    for name, got, exact in zip(("dx", "dw"), pol.gated_ffn_grad(dh, x, w, act=act), want):
        assert torch.isfinite(got).all() and float(exact.abs().max()) < torch.finfo(x.dtype).max, (what, name)
        off, once = (float((v.double().cpu() - exact).norm()) for v in (got, exact.to(x.dtype)))
        assert off <= 1.05 * once, (what, name, off / once)


@pytest.mark.parametrize("dtype,act", [(BF16, "silu"), (F16, "gelu")])
@pytest.mark.parametrize("rows,D,H", [(4, 136, 8200), (129, 256, 256), (300, 520, 136), (1025, 64, 72), (3000, 264, 520)])
def test_ffn_gradient_is_as_exact_as_rounding_once(pol, rows, D, H, dtype, act):
    rounded_once(pol, *ffn.make(rows, D, H, dtype, rows + H), act, f"{rows} {D} {H} {dtype}")


@pytest.mark.parametrize("rows", [3, 20, 150])
def test_ffn_gradient_of_large_values(pol, rows):
    """float16: gradients of the projections far beyond 65,504, of which the results are finite."""
    x, w, dh = ffn.make(rows, 64, 72, F16, rows)
    x, dh = x * 2.0**-7, (dh.float().clamp(-2, 2) * 30000).half()
    w = torch.stack((w[0] * 2.0**-7, w[1] * 512))
    g = d(dh) * (d(x) @ d(w[1]).t())
    assert float(g.abs().max()) > 4 * 65504
    rounded_once(pol, x, w, dh, "silu", f"{rows}")


@pytest.mark.parametrize("rows", [2, 500, 3000])
def test_ffn_gradient_of_small_values(pol, rows):
    """float16: gradients of the projections near the smallest values, of which the results are sums of many or large
    multiples."""
    x, w, dh = ffn.make(rows, 64, 520, F16, rows)
    rounded_once(pol, x * 64, w * 2.0**-4, (dh.float() * 2.0**-18).half(), "gelu", f"{rows}")
