"""What the sums of the head's gradient leave: long ones, and those in which a confident row's terms cancel."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from tests.policy_ref import BF16, E, F16, ROUNDOFF  # noqa: E402
from tests.test_gpu_policy_head import definition, make  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pol():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2407_04221_gb300 import policy
    return policy


def one_sign(rows, D, V, dtype):
    """Positive x and w, of which columns, rows and words are of different sizes, so that results lie anywhere between two
    values of the type.  All tokens are word 0, whose row of w is 0: of the others G has one sign."""
    gen = torch.Generator(device="cuda").manual_seed(rows + V)
    uniform = lambda *shape: torch.rand(*shape, generator=gen, device="cuda")  # noqa: E731
    column = 2.0**uniform(D)
    x = ((0.5 + uniform(rows, D)) * column * 2.0**uniform(rows, 1) / 4).to(dtype)
    w = (uniform(V, D) * column * 6 * uniform(V, 1) / D).to(dtype)
    w[0] = 0
    return x, w, torch.zeros(rows, dtype=torch.int64, device="cuda"), -torch.ones(rows, device="cuda")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,D,V", [(262144, 1024, 1024), (64, 4096, 100000)])
def test_long_sums_of_one_sign(pol, rows, D, V, dtype):
    """Terms of one sign: 262,144 of dw, 100,000 of dx.  At an addition a tensor core truncates sixteen products and the sum,
    together by some 2^-22.5 of the sum; one that grows evenly is half its last on average.  Of 512 terms, 32 additions,
    that is 2^-18.5 of the result; sums of those are rounded.  The mean error of N results beside it is that of their
    rounding, at most u each, (u / 3^1/2) / N^1/2 as root mean square, of which four are allowed, and 2^-20 for
    exponentials whose errors have one sign."""
    x, w, tok, dl = one_sign(rows, D, V, dtype)
    grads = pol.head_log_probs_grad(dl, x, w, tok, pol.head_log_probs(x, w, tok))
    want = definition(x, w, tok, dl)[1:3]
    for name, got, exact in zip(("dx", "dw"), grads, (want[0], want[1])):
        if name == "dw":
            got, exact = got[1:], exact[1:]
        off = float(((got.double() - exact) / exact).mean())
        assert abs(off) <= 2.0**-18 + 2.0**-20 + 4 * ROUNDOFF[dtype] / (3 * got.numel())**0.5, (name, off)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,D,V", [(300, 4096, 1500), (60000, 64, 520), (8200, 1024, 4100)])
def test_gradient_of_many_terms_is_as_exact_as_rounding_once(pol, rows, D, V, dtype):
    """As `test_gradient_is_as_exact_as_rounding_once`, of more terms: those of a sum that is truncated are 512 at most, less
    than 2^-17 of the result, and logits of D terms are made of parts of 256, whose truncation leaves
    2^-20 of |l| < 16 in the shares: 2^-16, 0.1 of float16's 0.3 x 2^-11; 1.005 in quadrature.  1.02 is allowed."""
    x, w, tok, dl = make(rows, D, V, dtype, rows + V)
    want = definition(x, w, tok, dl)[1:3]
    for name, got, exact in zip(("dx", "dw"), pol.head_log_probs_grad(dl, x, w, tok, pol.head_log_probs(x, w, tok)), want):
        off, once = (float((v.double() - exact).norm()) for v in (got, exact.to(dtype)))
        assert off <= 1.02 * once, (name, off / once)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows", [1, 5, 8, 9, 300])
@pytest.mark.parametrize("D", [1024, 2048])
def test_confident_rows(pol, rows, D, dtype):
    """Rows that are sure of their token to 1e-4 and less, of logits between 30 and 60.  Their entry of G is 1 - p, what the others
    leave of one: an error d of it adds d w_t to dx, which is read off along w_t.  The sum of exponentials is 1 and the
    others', rounded by 2^-24 at every addition to the one: 32 of a lane's, the other half's, of three teams and seven
    tiles, or of four warps and sixteen joins: 48.  All else is relative to 1 - p: logits by 2 `off` (sums of D terms)
    each, G as two values u^2, and dx's rounding, u of each of D values of random sign, in its direction."""
    V, gen = 2048, torch.Generator().manual_seed(rows + D)
    base = torch.randn(D, generator=gen) * (30 / D)**0.5
    words = torch.randn(V, D, generator=gen) / D**0.5
    tok = torch.randint(0, V, (rows,), generator=gen)
    sure = 18 + 3 * torch.rand(rows, 1, generator=gen)
    x = (base + sure * words[tok]).to(dtype).cuda()
    w, tok, dl = (base + words).to(dtype).cuda(), tok.cuda(), torch.full((rows,), -4096.0).cuda()
    _, want, _, g, l, logs, _ = definition(x, w, tok, dl)
    rest = -torch.expm1(logs.gather(1, tok[:, None]))[:, 0]
    assert float(l.amax(1).min()) > 30 and float(rest.max()) < 3e-4
    dx, _ = pol.head_log_probs_grad(dl, x, w, tok, pol.head_log_probs(x, w, tok))
    wt = w[tok].double()
    along = ((dx.double() - want) * wt).sum(1) / wt.square().sum(1) / 4096
    off = 2 * D * (x.double().abs() @ w.double().abs().t()).amax(1)
    u = ROUNDOFF[dtype]
    rounding = 4 * u * ((want * wt).square().sum(1).sqrt() / wt.square().sum(1) / 4096) + (2.0**-25 / 4096 if dtype == F16 else 0.0)
    assert (along.abs() <= 48 * E + rest * (4 * off * E + 1.01 * u * u) + rounding).all(), float((along.abs() / rest).max())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows", [3, 40])
def test_what_is_left_of_one(pol, rows, dtype):
    """Two words, exact logits x and 0: G of the token is what dx's first value is, 1 - p = 1 / (1 + e^x).  The sum 1 +
    e^-x is rounded by 2^-24; its logarithm and what follows by 2^-20 of 1 - p, which is rounded to the type."""
    at = (6 + torch.arange(rows) * (10.0 / rows)).to(dtype)
    x = torch.zeros(rows, 8, dtype=dtype)
    x[:, 0] = at
    w = torch.zeros(2, 8, dtype=dtype)
    w[0, 0] = 1
    x, w, tok, dl = x.cuda(), w.cuda(), torch.zeros(rows, dtype=torch.int64).cuda(), torch.full((rows,), 4096.0).cuda()
    dx, dw = pol.head_log_probs_grad(dl, x, w, tok, pol.head_log_probs(x, w, tok))
    rest = torch.sigmoid(-at.double())
    got = dx[:, 0].double().cpu() / 4096
    assert ((got - rest).abs() <= 1.01 * E + rest * (2.0**-20 + 1.01 * ROUNDOFF[dtype])).all()
    assert not dx[:, 1:].any()
