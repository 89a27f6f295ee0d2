"""What is not finite in the operators over cell words: in tables, logits, teachers, and places that do not count."""
from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")

from tests import test_gpu_policy_distill as dis  # noqa: E402
from tests.policy_ref import BF16, F16, F32  # noqa: E402
from tests.test_gpu_policy_head import make  # noqa: E402

pytestmark = pytest.mark.gpu
NAN, INF = math.nan, math.inf


@pytest.fixture(scope="module")
def pol():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2407_04221_gb300 import policy
    return policy


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows", [1, 7, 40, 256, 700])
def test_head_without_tokens(pol, rows, dtype):
    """Rows without a token add nothing to dw, whatever the table holds."""
    x, w, tok, dl = make(rows, 72, 500, dtype, rows)
    w[3], w[77, 5], w[499] = NAN, INF, -INF
    tok[:] = -1
    out = pol.head_log_probs(x, w, tok)
    assert not any(out[k].any() for k in out)
    dx, dw = pol.head_log_probs_grad(dl, x, w, tok, out)
    assert not dx.any() and not dw.any()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("count", [1, 3, 63, 64, 65, 200, 256, 300])
@pytest.mark.parametrize("absent", [0, 90])
def test_head_word_that_nothing_says(pol, count, absent, dtype):
    """A word of logit -inf in all rows: its share and its row of dw are 0, of any number of rows, with padding or without."""
    x, w, tok, dl = make(count + absent, 72, 500, dtype, count, 0.0)
    tok[count:] = -1
    x, tok = (v[torch.randperm(count + absent, generator=torch.Generator().manual_seed(count)).cuda()] for v in (x, tok))
    x[:, 5] = x[:, 5].abs() + 0.5
    tok[tok == 77] = 78
    w[77, 5] = -INF
    out = pol.head_log_probs(x, w, tok)
    assert all(torch.isfinite(out[k]).all() for k in out)
    _, dw = pol.head_log_probs_grad(dl, x, w, tok, out)
    assert not dw[77].any()
    assert torch.isfinite(dw).all()


@pytest.mark.parametrize("bad", [NAN, INF])
@pytest.mark.parametrize("rows", [3, 40])
def test_head_peaks(pol, rows, bad):
    """The largest logit: infinite where one is, else NaN where one is; both make logz and logp NaN."""
    x, w, tok, _ = make(rows, 64, 300, BF16, rows, 0.0)
    good = pol.head_log_probs(x, w, tok)
    x = x.abs() + 0.5
    w[7] = 0
    w[7, 3] = bad
    tok[tok == 7] = 8
    out = pol.head_log_probs(x, w, tok)
    assert torch.isnan(out["logz"]).all() and torch.isnan(out["logp"]).all()
    assert torch.equal(out["peak"].nan_to_num(1.0, 2.0, 3.0), torch.full_like(good["peak"], bad).nan_to_num(1.0, 2.0, 3.0))


SIZES = [5, 8, 9, 100, 1000, 1500, 5000, 33001]


def at_start(x, start):
    """The same rows, from elsewhere in 16 bytes."""
    wide = torch.zeros(x.shape[0], x.shape[1] + 9, dtype=x.dtype, device=x.device)
    wide[:, start:start + x.shape[1]] = x
    return wide[:, start:start + x.shape[1]]


@pytest.mark.parametrize("V", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("start", [None, 0, 1])
def test_distill_entries_that_are_not_there(pol, V, dtype, start):
    """Masked entries and those of logit -inf have no gradient, whatever else their row holds: NaN, +inf."""
    x, t, index, m, dkl = dis.make(1300 if V == 1500 else 40, V, 4, dtype, V, True, 0.0)
    x = x if start is None else at_start(x, start)
    x[:, 1::5], m[:, 2::7] = -INF, 0
    m[:, 0], x[:, 0] = 1, 1.0
    x[1, 0], x[3, 0], x[5, V - 1] = NAN, INF, NAN
    m[5, V - 1] = 1
    out = pol.distill(x, t, index, mask=m)
    got = pol.distill_grad(dkl, x, t, index, out, mask=m)
    gone = (m == 0) | (x == -INF)
    assert not got[gone].any()
    for r in (1, 3, 5):
        assert torch.isnan(got[r][~gone[r]]).all() and torch.isnan(out["kl"][r])
    keep = torch.isfinite(out["logz"])
    assert int(keep.sum()) == x.shape[0] - 3 and torch.isfinite(got[keep]).all()


@pytest.mark.parametrize("V", SIZES)
@pytest.mark.parametrize("bad", [NAN, INF])
def test_distill_bad_teachers(pol, V, bad):
    """A teacher's value that is NaN or +inf makes kl NaN, and the gradient of the entries that the row's alternatives name;
    the others have their share of it, as without a teacher's weight."""
    x, t, index, m, dkl = dis.make(1300 if V == 1500 else 40, V, 3, F32, V, gone=0.0)
    good = pol.distill(x, t, index)
    right = pol.distill_grad(dkl, x, t, index, good)
    t[1, 2], t[4, 0] = bad, bad
    out = pol.distill(x, t, index)
    got = pol.distill_grad(dkl, x, t, index, out)
    named = torch.zeros_like(x, dtype=torch.bool).scatter_(1, index.long(), True)
    bad_rows = torch.zeros_like(named[:, 0])
    bad_rows[[1, 4]] = True
    assert torch.equal(torch.isnan(out["kl"]), bad_rows) and torch.equal(torch.isnan(got), named & bad_rows[:, None])
    assert torch.equal(got[~(named & bad_rows[:, None])], right[~(named & bad_rows[:, None])])


@pytest.mark.parametrize("V", SIZES)
@pytest.mark.parametrize("heat", [1.0, 2.0])
def test_distill_weights_of_almost_nothing(pol, V, heat):
    """An alternative whose weight is above 0 in 32 bits, down to 2^-149, and that the student does not have makes kl
    infinite; one whose weight is 0 there does not."""
    x, t, index, _, dkl = dis.make(8, V, 2, F32, V, gone=0.0)
    index[:, 0], index[:, 1] = 0, 2
    below = torch.tensor([0.0, 20.0, 80.0, 88.0, 95.0, 102.0, 110.0, 1000.0], device="cuda") * heat
    t[:, 0], t[:, 1] = 3.0, 3.0 - below
    m = torch.ones(V, dtype=torch.uint8, device="cuda")
    m[2] = 0
    kl = pol.distill(x, t, index, temperature=heat, mask=m)["kl"]
    assert torch.isinf(kl[:6]).all() and torch.isfinite(kl[6:]).all()


@pytest.mark.parametrize("V", SIZES)
def test_distill_peaks(pol, V):
    """As the head's: infinite where a logit is, else NaN where one is, -inf where nothing is left."""
    x, t, index, _, _ = dis.make(40, V, 2, F32, V, gone=0.0)
    x[1, 2], x[3, 0], x[5], x[7, 1] = NAN, INF, -INF, -INF
    x[9, 1], x[9, 4] = NAN, INF
    out = pol.distill(x, t, index)
    want = x.amax(1)
    want[9] = INF
    assert torch.equal(out["peak"].nan_to_num(9.0, 1e30, -1e30), want.nan_to_num(9.0, 1e30, -1e30))
    assert torch.equal(torch.isnan(out["logz"]), torch.isnan(x).any(1) | (x == INF).any(1))
