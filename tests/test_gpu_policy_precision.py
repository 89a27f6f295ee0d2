"""What the policy operators' gradients may lose: no more than rounding the result once, whatever the sizes, and of
32-bit logits no more than the formula's own operations."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from tests import test_gpu_policy_ffn as ffn  # noqa: E402
from tests import test_gpu_policy_logp as logp  # noqa: E402
from tests.policy_ref import BF16, F16, F32, close, d, gated_ffn  # noqa: E402

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


# ------------------------------------------------------------ log probabilities

@pytest.mark.parametrize("rows,V", [(20000, 2), (20000, 5), (20000, 8), (5000, 20), (2000, 64), (500, 1000), (300, 3000),
                                    (1300, 3000), (3, 50000)])
@pytest.mark.parametrize("sure", [False, True])
def test_gradient_of_32_bit_logits(pol, rows, V, sure):
    """Against the formula of what the forward pass returned, in 64 bits.  With e = 2^-24: log p = (x - peak) - logz is
    off by e (|x - peak| + |log p|); its product with log2(e), itself rounded, by 2 e |log p| more; the exponential by
    2^-22 relatively: p by e (|x - peak| + 3 |log p| + 4).  c = dlogp + dentropy entropy is off by e (|c| + |dentropy
    entropy|), dentropy log p + c by e of itself and dentropy times log p's error more, their product with p by e."""
    x, tok, _, dl, de = logp.make(rows, V, F32, rows + V)
    if sure:  # of the token: p near one
        x[torch.arange(rows), tok] = x.amax(1) + 6 + 10 * torch.rand(rows, generator=torch.Generator().manual_seed(V)).cuda()
    out = pol.log_probs(x, tok)
    got = pol.log_probs_grad(dl, de, x, tok, out)
    low = d(x) - d(out["peak"])[:, None]
    lp, dl, de, H = low - d(out["logz"])[:, None], d(dl)[:, None], d(de)[:, None], d(out["entropy"])[:, None]
    p, c = lp.exp(), dl + de * H
    q = c + de * lp
    want = dl * (torch.arange(V) == tok.cpu()[:, None]) - p * q
    scale = p * (q.abs() * (low.abs() + 3 * lp.abs() + 6) + c.abs() + (de * H).abs() + de.abs() * (low.abs() + lp.abs()))
    close(got, want, 1.02 * scale, f"{rows}x{V}")
