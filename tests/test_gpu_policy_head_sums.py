"""What the sums of the head's gradient leave of terms that cancel: those of rows that are sure of their token."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

from tests.policy_ref import BF16, E, F16, ROUNDOFF  # noqa: E402
from tests.test_gpu_policy_head import definition  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pol():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2407_04221_gb300 import policy
    return policy


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
