"""Log probabilities, entropy, top alternatives and their gradient against the definition in 64 bits
(tests/policy_ref.py)."""
from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")

from tests import policy_ref as ref  # noqa: E402
from tests.policy_ref import BF16, E, F16, F32, close, d  # noqa: E402

pytestmark = pytest.mark.gpu
NAN, INF = math.nan, math.inf


@pytest.fixture(scope="module")
def pol():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2407_04221_gb300 import policy
    return policy


def make(rows, V, dtype, seed, tokens=torch.int64, scale=3.0):
    gen = torch.Generator().manual_seed(seed)
    x = (scale * torch.randn(rows, V, generator=gen)).to(dtype).cuda()
    tok = torch.randint(0, min(V, 256) if tokens == torch.uint8 else V, (rows,), generator=gen).to(tokens).cuda()
    mask = (torch.rand(rows, V, generator=gen) < 0.7).to(torch.uint8).cuda()
    dl, de = (torch.randn(rows, generator=gen).cuda() for _ in range(2))
    return x, tok, mask, dl, de


def check(pol, x, tok, mask, dl, de, top, what):
    """Bounds: exp(x - m) is good to (|x - m| + 4) e relatively, the sum of V of them, 32 or more at a time, to
    V / 32 + 16 roundings more; the row's spread R = max |x - m| over entries that count (beyond 104 they are 0)
    bounds all exponents.  logz is off by e (R + V / 32 + 24 + |logz|), a log probability by that and its own two
    roundings, the entropy by e (2 R + V / 32 + 32) (1 + R)."""
    V = x.shape[-1]
    rows = x.reshape(-1, V).shape[0]
    xd = d(x).reshape(-1, V).requires_grad_()
    td = tok.cpu().long().reshape(-1)
    md = None if mask is None else mask.cpu().expand(x.shape).reshape(-1, V)
    logp, entropy, peak, logz, logs, present = ref.log_probs(xd, td, md)
    out = pol.log_probs(x, tok, mask=mask, top=top)
    with torch.no_grad():
        wide = torch.where(present, peak[:, None] - xd, torch.zeros_like(xd)).amax(1)
        R = wide.clamp(max=104)
        g = R + V / 32 + 24
        near = g + torch.where(logz == -INF, torch.zeros_like(logz), logz).abs()
        lpn = near + wide  # (a log probability may be far below those that count)
    close(out["peak"].reshape(-1), peak, 0.0, what + " peak")
    close(out["logz"].reshape(-1), logz, near, what + " logz")
    close(out["logp"].reshape(-1), logp, 2 * lpn, what + " logp")
    close(out["entropy"].reshape(-1), entropy, (g + R) * (1 + R), what + " entropy")
    if top:
        index = ref.top_of(xd.detach(), present, top)
        assert torch.equal(out["top_index"].cpu().reshape(-1, top), index), what
        want = torch.where(index >= 0, logs.gather(1, index.long().clamp(min=0)), torch.full(index.shape, -INF).double())
        close(out["top_logp"].reshape(-1, top), want, 2 * lpn[:, None], what + " top")
    if dl is None:
        return out
    loss = torch.zeros((), dtype=torch.float64)
    live = present.any(1)
    ok = live & (logp.detach() != -INF)
    loss = loss + (torch.where(ok, logp, torch.zeros_like(logp)) * d(dl).reshape(-1)).sum()
    loss = loss + (torch.where(live, entropy, torch.zeros_like(entropy)) * d(de).reshape(-1)).sum()
    (want,) = torch.autograd.grad(loss, xd)
    want = torch.where(present, want, torch.zeros_like(want))
    with torch.no_grad():
        # a masked token still moves the others: dlogp (0 - p)
        lost = live & ~ok & (td >= 0) & (td < V)
        p = torch.where(present, logs, torch.full_like(logs, -INF)).exp()
        want = want - torch.where(lost, d(dl).reshape(-1), torch.zeros(rows).double())[:, None] * p
        la = torch.where(present, logs, torch.zeros_like(logs)).abs()
        dla, dea = d(dl).reshape(-1, 1).abs(), d(de).reshape(-1, 1).abs()
        rel = (2 * near + 8)[:, None] + la.clamp(max=104)
        scale = p * (dla + dea * (la + entropy[:, None])) * (rel + 8) + p * dea * (rel + ((g + R) * (1 + R))[:, None]) + 4 * dla * (td[:, None] == torch.arange(V))
    got = pol.log_probs_grad(dl, de, x, tok, out, mask=mask)
    close(got.reshape(-1, V), want, scale, what + " dlogits")
    return out


SIZES = [(1, 1), (3, 2), (1000, 5), (7, 17), (300, 31), (65, 32), (129, 33), (40, 100), (33, 256), (9, 1000), (6, 1023),
         (5, 1024), (4, 1025), (5, 4097), (3, 8192), (2, 20001), (2, 65536), (1, 70001)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,V", SIZES)
def test_log_probs(pol, rows, V, dtype):
    x, tok, mask, dl, de = make(rows, V, dtype, rows + V)
    check(pol, x, tok, None, dl, de, min(V, 8), f"{rows}x{V} {dtype}")
    check(pol, x, tok, mask, dl, de, min(V, 3), f"{rows}x{V} {dtype} masked")


@pytest.mark.parametrize("V", [5, 40, 1000, 30000])
@pytest.mark.parametrize("top", [0, 1, 5, 20, 32])
def test_top(pol, V, top):
    x, tok, mask, dl, de = make(12, V, F32, V + top)
    check(pol, x, tok, mask, None, None, min(top, V), f"top {top} of {V}")


@pytest.mark.parametrize("V", [5, 33, 1024, 5000, 40000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_ties_go_to_the_lowest_index(pol, V, dtype):
    """A row of one value, rows of few values, both zeros alike, the largest together at the end."""
    x, tok, _, dl, de = make(6, V, dtype, V)
    x[0] = 1.5
    x[1] = x[1].round().clamp(-1, 1)
    x[2] = torch.where(torch.arange(V, device="cuda") % 2 == 0, 0.0, -0.0).to(dtype)
    x[3, -min(V, 70):] = 20.0
    x[4, ::3] = 20.0
    x[5] = torch.arange(V, 0, -1, device="cuda").to(dtype)
    check(pol, x, tok, None, dl, de, min(V, 32), f"ties of {V}")


@pytest.mark.parametrize("V", [4, 5, 37, 300, 3000])
def test_rows_with_nothing_left(pol, V):
    """Masked out, -inf throughout, the type's lowest value throughout, and one entry left."""
    x, tok, mask, dl, de = make(8, V, F32, V)
    mask[1] = 0
    x[2] = -INF
    x[3] = torch.finfo(F32).min
    mask[4] = 0
    mask[4, V // 2] = 1
    x[5, : V - 1] = -INF
    mask[5] = 1
    tok[5] = V - 1
    out = check(pol, x, tok, mask, dl, de, min(V, 4), "nothing left")
    assert out["peak"][1] == out["logz"][1] == -INF and out["logp"][1] == -INF and out["entropy"][1] == 0
    assert (out["top_index"][[1, 2]] == -1).all()


@pytest.mark.parametrize("V", [5, 50, 2000])
def test_masked_places_may_hold_anything(pol, V):
    x, tok, mask, dl, de = make(20, V, F32, V)
    clean = pol.log_probs(x, tok, mask=mask, top=min(V, 5))
    grad = pol.log_probs_grad(dl, de, x, tok, clean, mask=mask)
    for bad in (NAN, INF, -INF, 3e38):
        y = torch.where(mask != 0, x, torch.full_like(x, bad))
        got = pol.log_probs(y, tok, mask=mask, top=min(V, 5))
        assert all(torch.equal(got[k], clean[k]) for k in clean), bad
        assert torch.equal(pol.log_probs_grad(dl, de, y, tok, got, mask=mask), grad), bad


@pytest.mark.parametrize("V", [5, 90, 3000])
def test_bad_values_stay_in_their_row(pol, V):
    x, tok, mask, dl, de = make(30, V, F32, V)
    clean = pol.log_probs(x, tok, top=min(V, 5))
    x[4, 1], x[9, 0] = NAN, INF
    got = pol.log_probs(x, tok, top=min(V, 5))
    keep = [r for r in range(30) if r not in (4, 9)]
    for k in clean:
        assert torch.equal(got[k][keep], clean[k][keep])
    assert torch.isnan(got["logz"][[4, 9]]).all() and torch.isnan(got["entropy"][[4, 9]]).all()
    assert int(got["top_index"][4, 0]) == 1 and int(got["top_index"][9, 0]) == 0


@pytest.mark.parametrize("V", [5, 70, 2000])
@pytest.mark.parametrize("tokens", [torch.uint8, torch.int32, torch.int64])
def test_token_types_and_absent_tokens(pol, V, tokens):
    x, tok, mask, dl, de = make(64, V, BF16, V, tokens)
    if tokens == torch.uint8:
        tok[::5] = 255 if V < 256 else 0
    else:
        tok[::5], tok[1::7] = -1, V
    check(pol, x, tok, mask, dl, de, 2, f"{tokens}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [5, 40, 1000, 5000])
def test_strides_and_starts(pol, V, dtype):
    """Rows of a wider array from an odd start, three axes, one row and one mask for all."""
    x, tok, mask, dl, de = make(24, V + 5, dtype, V)
    tok = tok.clamp(max=V - 1)
    check(pol, x[:, 1:V + 1], tok, mask[:, 3:V + 3], dl, de, 3, "offset")
    check(pol, x[:, :V].unflatten(0, (4, 6)), tok.reshape(4, 6), None, dl.reshape(4, 6), de.reshape(4, 6), 3, "axes")
    check(pol, x[:1, :V].expand(24, V), tok, mask[0, :V].contiguous(), dl, de, 3, "one for all")
    check(pol, x[::2, :V], tok[::2].contiguous(), mask[::2, :V], dl[::2].contiguous(), de[::2].contiguous(), 3, "second")


@pytest.mark.parametrize("V", [5, 3000])
def test_one_gradient_alone(pol, V):
    x, tok, mask, dl, de = make(10, V, F32, V)
    out = pol.log_probs(x, tok, mask=mask)
    zero = torch.zeros_like(dl)
    both = [pol.log_probs_grad(a, b, x, tok, out, mask=mask) for a, b in ((dl, zero), (zero, de))]
    assert torch.equal(both[0], pol.log_probs_grad(dl, None, x, tok, dict(out, entropy=None), mask=mask))
    assert torch.equal(both[1], pol.log_probs_grad(None, de, x, tok, out, mask=mask))


def test_large_logits(pol):
    """Logits near the type's limits: differences, not the values, are exponentiated."""
    x, tok, mask, dl, de = make(30, 600, F32, 1)
    check(pol, x + 1e4, tok, mask, dl, de, 4, "shifted")
    check(pol, x * 40, tok, mask, dl, de, 4, "wide")


def test_no_rows(pol):
    x, tok, mask, dl, de = make(0, 7, F32, 1)
    out = pol.log_probs(x, tok, top=2)
    assert out["logp"].shape == (0,) and out["top_index"].shape == (0, 2)
    assert pol.log_probs_grad(dl, de, x, tok, out).shape == (0, 7)


@pytest.mark.parametrize("V", [5, 200, 5000])
def test_gradient_against_differences(pol, V):
    """Central differences of the kernel's own forward pass in f32 along unit directions, step 2^-4: the loss's third
    derivative there is at most |dl| + |de| (1 + entropy) per row, so truncation is below 2^-10 of that; rounding adds
    e / step of the outputs' magnitudes."""
    x, tok, mask, dl, de = make(8, V, F32, V)
    out = pol.log_probs(x, tok)
    grad = pol.log_probs_grad(dl, de, x, tok, out)
    u = torch.randn(x.shape, generator=torch.Generator().manual_seed(V))
    u = (u / u.norm()).cuda()
    step, side = 2.0**-4, []
    for s in (step, -step):
        o = pol.log_probs(x + s * u, tok)
        side.append(float((o["logp"].double() * dl.double() + o["entropy"].double() * de.double()).sum()))
    slope, want = (side[0] - side[1]) / (2 * step), float((grad.double() * u.double()).sum())
    size = float((dl.abs() * (out["logp"].abs() + 4) + de.abs() * (1 + out["entropy"])).double().sum())
    assert abs(slope - want) <= 0.01 * float(grad.double().norm()) + 2.0**-10 * size / 8 + 16 * E / step * size
