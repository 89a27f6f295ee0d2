"""The gated recurrence and its gradient against the definition in 64 bits, step by step (tests/policy_ref.py)."""
from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")

from tests import policy_ref as ref  # noqa: E402
from tests.policy_ref import BF16, E, F16, F32, close, d  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pol():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2407_04221_gb300 import policy
    return policy


def make(T, B, D, dtype, resets, seed, shift=1.0):
    gen = torch.Generator().manual_seed(seed)
    g = (1.5 * torch.randn(T, B, D, generator=gen) + shift).to(dtype).cuda()
    v, dh = (torch.randn(T, B, D, generator=gen).to(dtype).cuda() for _ in range(2))
    reset = None if resets is None else (torch.rand(T, B, generator=gen) < resets).to(torch.uint8).cuda()
    h0, dlast = (torch.randn(B, D, generator=gen).cuda() for _ in range(2))
    return g, v, reset, h0, dh, dlast


def check(pol, g, v, reset, h0, dh, dlast, what):
    """Bounds: a gate and its complement are good to 8 e (argument in the exponent: |g| e more) relatively.  A step
    adds at most (|g| + 16) e of the magnitudes m_t = a m_{t-1} + (1 - a) |v| there, which later steps weigh by their
    gates just as they weigh m; a state is a convex mix, so its error is at most e (|g|max + 16) S with S the largest
    magnitude so far times 1 / (1 - a) summed up, bounded here by the same recurrence on the errors themselves."""
    gd, vd = d(g).requires_grad_(), d(v).requires_grad_()
    hd = None if h0 is None else d(h0).requires_grad_()
    rd = None if reset is None else reset.cpu()
    h, last = ref.scan(gd, vd, rd, hd)
    got_h, got_last, states = pol.scan(g, v, reset, h0, save=True)
    with torch.no_grad():
        unit = gd.abs().clamp(max=88) + 16
        a, z = torch.sigmoid(gd), torch.sigmoid(-gd)
        keep = torch.ones(g.shape[:2]) if rd is None else (rd == 0).double()
        err, mag = torch.zeros(g.shape[1:]).double(), (torch.zeros(g.shape[1:]).double() if h0 is None else d(h0).abs())
        errs, mags, herr = [], [], []  # of the state that a step starts from, and of the one that it leaves
        for t in range(g.shape[0]):
            k = keep[t][:, None]
            mags.append(mag * k)
            errs.append(err * k)
            step = a[t] * k * mag + z[t] * vd[t].abs()
            err, mag = a[t] * k * err + unit[t] * step, step
            herr.append(err)
        herr = torch.stack(herr)
    close(got_h, h, herr, what + " h")
    close(got_last, last, herr[-1], what + " last")
    plain = pol.scan(g, v, reset, h0)
    assert torch.equal(plain[0], got_h) and torch.equal(plain[1], got_last), what
    ins = [gd, vd] + ([hd] if hd is not None else [])
    loss = (h * d(dh)).sum() + (0 if dlast is None else (last * d(dlast)).sum())
    want = torch.autograd.grad(loss, ins)
    dgate, dvalue, dh0 = pol.scan_grad(dh, g, v, reset, states, dlast=dlast)
    with torch.no_grad():
        l = torch.zeros(g.shape[1:]).double() if dlast is None else d(dlast).abs()
        le = torch.zeros_like(l)
        gscale, vscale = torch.empty_like(a), torch.empty_like(a)
        for t in reversed(range(g.shape[0])):
            l = l + d(dh[t]).abs()
            le = le + 2 * l
            held = mags[t] + vd[t].abs()
            vscale[t] = z[t] * (le + unit[t] * l)
            gscale[t] = a[t] * z[t] * (le * held + l * errs[t] + 3 * unit[t] * l * held)
            k = keep[t][:, None]
            le = a[t] * k * (le + unit[t] * l)
            l = a[t] * k * l
    close(dgate, want[0], gscale, what + " dgate")
    close(dvalue, want[1], vscale, what + " dvalue")
    if hd is not None:
        close(dh0, want[2], le, what + " dh0")


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T,B,D", [(1, 1, 1), (1, 700, 33), (2, 3, 5), (15, 2, 64), (16, 4, 32), (17, 5, 31),
                                   (33, 2, 130), (64, 3, 64), (65, 2, 100), (128, 3, 256), (129, 1, 96), (300, 2, 72)])
@pytest.mark.parametrize("resets", [None, 0.05])
def test_scan(pol, T, B, D, dtype, resets):
    check(pol, *make(T, B, D, dtype, resets, T * B * D), f"{T}x{B}x{D} {dtype}")


@pytest.mark.parametrize("T,B,D,dtype", [(1021, 1, 40, F32), (4097, 1, 7, BF16), (9001, 1, 64, F32),
                                         (2500, 3, 130, BF16), (5000, 2, 66, F16)])
@pytest.mark.parametrize("resets", [0.0, 0.002])
def test_long(pol, T, B, D, dtype, resets):
    """Sequences of many chunks; gates near one carry a state over several of them."""
    check(pol, *make(T, B, D, dtype, resets, T, shift=4.0), f"{T}x{B}x{D}")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_and_starts(pol, dtype):
    """Sequence-first arrays, rows of a wider array from odd starts, a gate for all steps and one for all sequences."""
    T, B, D = 70, 6, 48
    g, v, reset, h0, dh, dlast = make(T, B, D + 9, dtype, 0.05, 1)
    h0, dlast = h0[:, :D].contiguous(), dlast[:, :D].contiguous()
    swap = [x[..., :D].transpose(0, 1).contiguous().transpose(0, 1) for x in (g, v, dh)]
    check(pol, swap[0], swap[1], reset.t().contiguous().t(), h0, swap[2], dlast, "sequence first")
    check(pol, g[..., 1:D + 1], v[..., 8:D + 8], reset, h0, dh[..., 3:D + 3], dlast, "odd starts")
    one = g[:1, :, :D].expand(T, B, D)
    check(pol, one, v[..., :D], reset, h0, dh[:, :1, :D].expand(T, B, D), dlast, "one for all steps")
    check(pol, g[:, :1, :D].expand(T, B, D), v[..., :D], reset[:, :1].expand(T, B), h0, dh[..., :D], None, "one for all")


@pytest.mark.parametrize("T", [5, 400])
def test_without_state_and_reset_everywhere(pol, T):
    g, v, reset, h0, dh, dlast = make(T, 3, 40, F32, 0.1, T)
    check(pol, g, v, reset, None, dh, None, "no state")
    check(pol, g, v, torch.full_like(reset, 255), h0, dh, dlast, "reset at every step")
    check(pol, g, v, reset.bool(), h0, dh, dlast, "bool")


@pytest.mark.parametrize("dtype", [F32, F16])
def test_saturated_gates(pol, dtype):
    """Gates far out: 0 and 1 to the last bit, and the complement without cancellation."""
    g, v, reset, h0, dh, dlast = make(200, 2, 64, dtype, 0.02, 9)
    g[::3] = 30.0
    g[1::7] = -40.0
    check(pol, g, v, reset, h0, dh, dlast, "saturated")
    g[::3], g[1::7] = math.inf, -math.inf
    h, last = pol.scan(g, v, reset, h0)
    want, wlast = ref.scan(d(g), d(v), reset.cpu(), d(h0))
    close(h, want, 2000.0 * 4, "infinite gates")


@pytest.mark.parametrize("T", [40, 1500])
def test_reset_forgets_bad_values(pol, T):
    """NaN and infinity before an episode's begin are not seen after it, nor their gradients before it."""
    g, v, reset, h0, dh, dlast = make(T, 2, 33, F32, None, T)
    reset = torch.zeros(T, 2, dtype=torch.uint8, device="cuda")
    cut = T // 2
    reset[cut] = 1
    base = pol.scan(g, v, reset, h0, save=True)
    grad = pol.scan_grad(dh, g, v, reset, base[2], dlast=dlast)
    v2, dh2 = v.clone(), dh.clone()
    v2[cut - 3, 0, 5], v2[2, 1, 1] = float("nan"), float("inf")
    out = pol.scan(g, v2, reset, h0, save=True)
    assert torch.equal(out[0][cut:], base[0][cut:]) and torch.equal(out[1], base[1])
    assert torch.isnan(out[0][cut - 1, 0, 5]) and torch.isinf(out[0][2, 1, 1])
    dh2[cut + 1, 0, 5] = float("nan")
    got = pol.scan_grad(dh2, g, v, reset, base[2], dlast=dlast)
    assert torch.equal(got[0][:cut], grad[0][:cut]) and torch.equal(got[1][:cut], grad[1][:cut])
    assert torch.equal(got[2], grad[2]) and torch.isnan(got[1][cut, 0, 5])


def test_no_steps(pol):
    g = torch.empty(0, 3, 8, device="cuda")
    h0 = torch.randn(3, 8, device="cuda")
    h, last, states = pol.scan(g, g, None, h0, save=True)
    assert h.shape == (0, 3, 8) and torch.equal(last, h0)
    _, _, dh0 = pol.scan_grad(g, g, g, None, states, dlast=h0)
    assert torch.equal(dh0, h0)
    h, last = pol.scan(torch.empty(4, 0, 8, device="cuda"), torch.empty(4, 0, 8, device="cuda"))
    assert h.shape == (4, 0, 8) and last.shape == (0, 8)


def test_steps_one_by_one_match_the_whole(pol):
    """Acting one step at a time and reading the trajectory at once: the same states but for the order of
    multiplications (a bound of 40 steps' roundings)."""
    g, v, reset, h0, dh, dlast = make(40, 5, 64, F32, 0.1, 2)
    whole, last = pol.scan(g, v, reset, h0)
    state = h0
    for t in range(40):
        h, state = pol.scan(g[t:t + 1], v[t:t + 1], reset[t:t + 1], state)
        close(h[0], d(whole[t]), 40 * 24 * 4.0, f"step {t}")


def test_gradient_against_differences(pol):
    """Central differences of the kernel's own forward pass in f32, along unit directions with a step of 2^-4: the
    loss's third derivative along a gate direction is below |loss terms|, so truncation stays below 2^-9 of |c| sqrt(T);
    rounding adds e / 2^-4 of the loss's magnitude."""
    g, v, reset, h0, dh, dlast = make(150, 2, 20, F32, 0.02, 4)
    h, last, states = pol.scan(g, v, reset, h0, save=True)
    grads = pol.scan_grad(dh, g, v, reset, states, dlast=dlast)
    gen = torch.Generator().manual_seed(1)
    step = 2.0**-4
    args = [g, v, h0]
    for k in range(3):
        u = torch.randn(args[k].shape, generator=gen)
        u = (u / u.norm()).cuda()
        side = []
        for s in (step, -step):
            moved = list(args)
            moved[k] = args[k] + s * u
            hh, ll = pol.scan(moved[0], moved[1], reset, moved[2])
            side.append(float((hh.double() * dh.double()).sum() + (ll.double() * dlast.double()).sum()))
        slope, want = (side[0] - side[1]) / (2 * step), float((grads[k].double() * u.double()).sum())
        assert abs(slope - want) <= 0.01 * float(grads[k].double().norm()) + 8 * E / step * float((h * dh).abs().double().sum())


def test_same_bits_again(pol):
    g, v, reset, h0, dh, dlast = make(6000, 2, 96, BF16, 0.001, 5, shift=4.0)
    first = pol.scan(g, v, reset, h0, save=True)
    back = pol.scan_grad(dh, g, v, reset, first[2], dlast=dlast)
    for _ in range(5):
        assert all(torch.equal(p, q) for p, q in zip(first[:2], pol.scan(g, v, reset, h0)))
        assert all(torch.equal(p, q) for p, q in zip(back, pol.scan_grad(dh, g, v, reset, first[2], dlast=dlast)))
