"""The policy operators at the sizes and layouts between which they change their way, against the definitions in 64 bits:
the bounds are those of the operators' own tests, whose `check` functions derive them."""
from __future__ import annotations

import gc
import threading

import pytest

torch = pytest.importorskip("torch")

from tests import test_gpu_policy_ffn as ffn  # noqa: E402
from tests import test_gpu_policy_logp as logp  # noqa: E402
from tests import test_gpu_policy_norm as norm  # noqa: E402
from tests import test_gpu_policy_scan as scan  # noqa: E402
from tests.policy_ref import (BF16, E, F16, F32, ROUNDOFF, SMALLEST, activate, close, d,  # noqa: E402
                              gated_ffn, top_of)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pol():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2407_04221_gb300 import policy
    return policy


def shifted(x):
    """x in a place that is aligned to one value only."""
    return torch.cat((x.new_zeros(1), x.reshape(-1)))[1:].view(x.shape)


# ------------------------------------------------------------ recurrence

@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T,B,D", [(2, 64, 64), (3, 130, 33), (4, 4100, 1), (5, 600, 7), (8, 65, 64), (8, 4096, 1),
                                   (9, 64, 65), (12, 130, 32), (16, 70, 61), (17, 64, 64)])
@pytest.mark.parametrize("resets", [None, 0.2])
def test_scan_of_few_steps_of_many_channels(pol, T, B, D, dtype, resets):
    scan.check(pol, *scan.make(T, B, D, dtype, resets, T * B + D), f"{T}x{B}x{D} {dtype}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [6, 14])
def test_scan_of_few_steps_strided(pol, T, dtype):
    B, D = 80, 64
    g, v, reset, h0, dh, dlast = scan.make(T, B, D + 9, dtype, 0.2, T)
    h0, dlast = h0[:, :D].contiguous(), dlast[:, :D].contiguous()
    swap = [x[..., :D].transpose(0, 1).contiguous().transpose(0, 1) for x in (g, v, dh)]
    scan.check(pol, swap[0], swap[1], reset.t().contiguous().t(), h0, swap[2], dlast, "sequence first")
    scan.check(pol, g[..., 1:D + 1], v[..., 8:D + 8], reset, h0, dh[..., 3:D + 3], dlast, "odd starts")
    scan.check(pol, g[:1, :, :D].expand(T, B, D), v[..., :D], reset, None, dh[:, :1, :D].expand(T, B, D), None, "broadcast")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,B,D", [(1, 8, 64), (6, 64, 64), (40, 3, 64), (300, 2, 66), (2000, 1, 64)])
def test_scan_states_aligned_to_one_value(pol, T, B, D, dtype):
    g, v, reset, h0, dh, dlast = scan.make(T, B, D, dtype, 0.01, T)
    scan.check(pol, g, v, reset, shifted(h0), dh, shifted(dlast), "states")
    scan.check(pol, *(shifted(x) for x in (g, v, reset, h0, dh, dlast)), "everything")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [31, 32, 33, 63, 64, 65, 127, 128, 129, 192, 193, 255, 256, 257, 1023, 1024, 1025, 1089])
def test_scan_at_the_ends_of_runs_and_chunks(pol, T, dtype):
    scan.check(pol, *scan.make(T, 2, 72, dtype, 0.02, T), f"{T} {dtype}")


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("D", [64, 66, 33, 1])
def test_scan_in_segments(pol, D, dtype):
    """Long sequences of few channels: by tensor copies, in pairs and one by one."""
    g, v, reset, h0, dh, dlast = scan.make(3001, 2, D, dtype, 0.001, D, shift=4.0)
    scan.check(pol, g, v, reset, h0, dh, dlast, f"{D}")
    wide = [torch.nn.functional.pad(x, (3, 2))[..., 3:3 + D] for x in (g, v, dh)]
    scan.check(pol, wide[0], wide[1], None, None, wide[2], None, f"{D} strided")


# ------------------------------------------------------------ log probabilities

@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,V", [(151, 1500), (152, 1500), (200, 1025), (160, 4096), (155, 4097), (152, 8191), (153, 8193)])
def test_log_probs_of_many_wide_rows(pol, rows, V, dtype):
    x, tok, mask, dl, de = logp.make(rows, V, dtype, rows + V)
    logp.check(pol, x, tok, mask, dl, de, 5, f"{rows}x{V} masked")
    logp.check(pol, x, tok, None, dl, de, 0, f"{rows}x{V}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [1500, 5001])
def test_log_probs_of_many_wide_rows_with_ties_and_gaps(pol, V, dtype):
    x, tok, mask, dl, de = logp.make(160, V, dtype, V)
    x[:40] = x[:40].round().clamp(-1, 1)
    x[40] = 1.5
    x[41, -70:] = 20.0
    x[42] = float("-inf")
    x[43] = torch.finfo(dtype).min
    mask[44] = 0
    mask[45] = 0
    mask[45, V - 1] = 1
    logp.check(pol, x, tok, mask, dl, de, 32, f"{V}")


@pytest.mark.parametrize("V", [100, 1500])
def test_log_probs_of_rows_from_odd_starts(pol, V):
    x, tok, mask, dl, de = logp.make(160, V + 9, BF16, V)
    tok = tok % V
    for k in (1, 3, 8):
        logp.check(pol, x[:, k:k + V], tok, mask[:, k:k + V], dl, de, 3, f"{V} from {k}")
    logp.check(pol, x[:1, 1:V + 1].expand(160, V), tok, mask[0, :V].contiguous(), dl, de, 3, f"{V} one row for all")


# ------------------------------------------------------------ layer norm

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,n", [(3001, 257), (3001, 513), (2500, 1029), (1501, 2051), (700, 4805), (400, 8193), (320, 16383)])
def test_norm_of_many_rows_from_odd_starts(pol, rows, n, dtype):
    x, dy, w, b = norm.make(rows, n + 8, dtype, F32, n)
    w, b = w[:n].contiguous(), b[:n].contiguous()
    for k in (0, 1, 5):
        norm.check(pol, x[:, k:k + n], dy[:, 7 - k:7 - k + n], w, b, f"{rows}x{n} from {k}")
    norm.check(pol, x[:, :n].contiguous(), dy[:, :n].contiguous(), w, b, f"{rows}x{n}")


# ------------------------------------------------------------ gated feed-forward

@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,D,H", [(3, 264, 1000), (4, 256, 512), (4, 1032, 72), (5, 256, 512), (16, 1024, 264)])
def test_ffn_of_few_rows(pol, rows, D, H, dtype):
    x, w, dh = ffn.make(rows, D, H, dtype, rows + D)
    ffn.check(pol, x, w, dh, "silu", f"{rows} {D} {H}")
    ffn.check(pol, x, w, dh, "gelu", f"{rows} {D} {H}")


# ------------------------------------------------------------ calls

def test_calls_from_two_threads(pol):
    """Calls let go of the interpreter: two threads on streams of their own get what one gets."""
    sets = [norm.make(300, 1000, BF16, F32, k) for k in range(2)]
    want = [pol.layer_norm(x, w, b) for x, _, w, b in sets]
    torch.cuda.synchronize()
    wrong = []

    def work(k):
        x, _, w, b = sets[k]
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(200):
                got = pol.layer_norm(x, w, b)
                if not all(torch.equal(p, q) for p, q in zip(got, want[k])):
                    wrong.append(k)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_calls_keep_nothing(pol):
    """Memory is as before after calls, refused ones among them; parameters that want gradients are taken as they are."""
    x, dy, w, b = norm.make(64, 520, BF16, F32, 1)
    p = torch.nn.Parameter(w)
    tok = torch.zeros(64, dtype=torch.int64, device="cuda")
    torch.cuda.synchronize()
    gc.collect()  # (cycles that tests before this one left)
    before = torch.cuda.memory_allocated()
    for k in range(50):
        y, mean, rstd = pol.layer_norm(x, p, b)
        out = pol.log_probs(x, tok, top=3)
        with pytest.raises(ValueError):
            pol.layer_norm(x, p, b[:9])
        with pytest.raises(ValueError):
            pol.log_probs_grad(mean, None, x, tok, dict(out, peak=None))
        with pytest.raises(TypeError):
            pol.layer_norm(x, p, b, eps="small")
        with pytest.raises(TypeError):
            pol.log_probs(x, tok, top="all")
    assert not y.requires_grad
    del y, mean, rstd, out  # (dy stays: it was there before)
    assert dy.shape == x.shape
    assert torch.cuda.memory_allocated() == before


# ------------------------------------------------------------ enough rows for another way

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,V,top", [(607, 1500, 3), (608, 1025, 5), (640, 2049, 0), (608, 8191, 0), (1216, 8193, 0),
                                        (1217, 1500, 2), (1300, 4095, 0), (1216, 4097, 0)])
def test_log_probs_of_very_many_wide_rows(pol, rows, V, top, dtype):
    x, tok, mask, dl, de = logp.make(rows, V, dtype, rows + V)
    logp.check(pol, x, tok, mask, dl, de, top, f"{rows}x{V} masked")
    logp.check(pol, x, tok, None, dl, de, 0, f"{rows}x{V}")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_log_probs_of_very_many_wide_rows_with_ties_and_gaps(pol, dtype):
    V = 1500
    x, tok, mask, dl, de = logp.make(1220, V, dtype, V)
    x[:40] = x[:40].round().clamp(-1, 1)
    x[40] = 1.5
    x[41, -70:] = 20.0
    x[42] = float("-inf")
    x[43] = torch.finfo(dtype).min
    mask[44] = 0
    mask[45] = 0
    mask[45, V - 1] = 1
    logp.check(pol, x, tok, mask, dl, de, 32, f"{V}")
    wide, wm = torch.nn.functional.pad(x, (3, 2)), torch.nn.functional.pad(mask, (3, 2))
    logp.check(pol, wide[:, 3:3 + V], tok, wm[:, 3:3 + V], dl, de, 0, f"{V} from 3")


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("V", [4, 6, 7, 8])
def test_log_probs_of_few_entries(pol, V, dtype):
    x, tok, mask, dl, de = logp.make(3001, V, dtype, V)
    mask[5] = 0
    x[6] = float("-inf")
    logp.check(pol, x, tok, mask, dl, de, V, f"{V}")
    logp.check(pol, torch.nn.functional.pad(x, (1, 2))[:, 1:1 + V], tok, mask, dl, de, 1, f"{V} from 1")


@pytest.mark.parametrize("rows,n", [(1, 300), (40, 384), (700, 512), (3001, 768), (500, 1000), (3001, 1024)])
def test_norm_of_whole_packs_of_floats(pol, rows, n):
    x, dy, w, b = norm.make(rows, n, F32, F32, n)
    norm.check(pol, x, dy, w, b, f"{rows}x{n}")
    norm.check(pol, x, dy, w.bfloat16(), b.bfloat16(), f"{rows}x{n}")
    x, dy, w, b = norm.make(rows, n + 4, F32, F32, n)
    norm.check(pol, x[:, 4:], dy[:, :n], w[:n].contiguous(), None, f"{rows}x{n} from 4")
    norm.check(pol, x[:, 3:3 + n], dy[:, 1:n + 1], w[:n].contiguous(), None, f"{rows}x{n} from 3")


@pytest.mark.parametrize("dtype,B", [(BF16, 101), (BF16, 102), (F32, 101), (F32, 152), (F32, 153)])
def test_scan_where_cutting_ends(pol, dtype, B):
    scan.check(pol, *scan.make(700, B, 64, dtype, 0.002, B, shift=3.0), f"{B} {dtype}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [190, 256, 384, 400, 512, 700, 900])
@pytest.mark.parametrize("B", [1, 38, 57])
def test_scan_of_few_chunks_in_segments(pol, T, B, dtype):
    scan.check(pol, *scan.make(T, B, 64, dtype, 0.005, T + B, shift=3.0), f"{T}x{B} {dtype}")


# ------------------------------------------------------------ few gradients of the projections, as two values each

def check_in_two(pol, x, w, dh, act, what):
    """The bounds of the operator's own tests, but for the rounding of the projections' gradients: a value and what it
    leaves, each rounded to u, are off by u^2 of the value and half the type's smallest step."""
    u, D, H, rows = ROUNDOFF[x.dtype], x.shape[1], w.shape[1], x.shape[0]
    xd, wd, dhd = d(x).requires_grad_(), d(w).requires_grad_(), d(dh)
    want = torch.autograd.grad((gated_ffn(xd, wd, act) * dhd).sum(), [xd, wd])
    xd, wd = xd.detach(), wd.detach()
    g, up = (xd @ wd[0].t()).requires_grad_(), xd @ wd[1].t()
    f = activate(g, act)
    (slope,) = torch.autograd.grad(f.sum(), g)
    g, f = g.detach(), f.detach()
    ge, ue = (2 * D * (xd.abs() @ wd[k].abs().t()) for k in (0, 1))
    fe = 1.13 * ge + (g.abs() + 16) * (f.abs() + 1e-3)
    a = dhd.abs()
    dg, du = a * up.abs() * slope.abs(), a * f.abs()
    dge, due = a * (ue * 1.13 + up.abs() * (0.8 * ge + g.abs() + 24)), a * fe
    er = [1.01 * u * u * v + SMALLEST[x.dtype] + E * e for v, e in ((dg, dge), (du, due))]
    dx, dw = pol.gated_ffn_grad(dh, x, w, act=act)
    wa, xa = wd.abs(), xd.abs()
    close(dx, want[0], 8 * H * (dg @ wa[0] + du @ wa[1]), what + " dx", er[0] @ wa[0] + er[1] @ wa[1])
    close(dw, want[1], 4 * rows * torch.stack((dg.t() @ xa, du.t() @ xa)), what + " dw",
          torch.stack((er[0].t() @ xa, er[1].t() @ xa)))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows,D,H", [(1, 64, 64), (1, 8, 8), (2, 1608, 144), (3, 72, 1000), (4, 64, 8192), (5, 520, 72),
                                      (17, 64, 64), (63, 72, 40), (64, 128, 256), (65, 72, 504), (128, 64, 256),
                                      (500, 40, 64)])
def test_ffn_gradient_of_few_is_rounded_once(pol, rows, D, H, dtype, act):
    assert rows * H <= 32768
    x, w, dh = ffn.make(rows, D, H, dtype, rows + D + H)
    check_in_two(pol, x, w, dh, act, f"{rows} {D} {H}")


@pytest.mark.parametrize("rows,H", [(4, 8200), (129, 256), (129, 248), (1025, 32), (1024, 32)])
def test_ffn_gradient_on_either_side_of_few(pol, rows, H):
    x, w, dh = ffn.make(rows, 136, H, BF16, rows)
    ffn.check(pol, x, w, dh, "silu", f"{rows} {H}")
    wide = torch.nn.functional.pad(x, (8, 16)), torch.nn.functional.pad(dh, (16, 8))
    ffn.check(pol, wide[0][:, 8:144], w, wide[1][:, 16:16 + H], "gelu", f"{rows} {H} strided")


@pytest.mark.parametrize("rows", [3, 6])
def test_ffn_gradient_beyond_the_type_is_infinite(pol, rows):
    """A projection's gradient of 60,000 x 4 x 0.93 is infinite in f16, and the input's with it, not NaN."""
    x, w, dh = ffn.make(rows, 64, 72, F16, rows)
    x[0], dh[0] = 0, 0
    x[0, 0], dh[0, 0] = 1, 60000
    w[:, 0] = 0.5
    w[0, 0, 0], w[1, 0, 0] = 1, 4
    dx, _ = pol.gated_ffn_grad(dh, x, w)
    assert torch.isinf(dx[0]).all() and torch.isfinite(dx[1:]).all()


def test_ffn_gradient_of_few_again(pol):
    x, w, dh = ffn.make(7, 264, 520, BF16, 5)
    first = pol.gated_ffn_grad(dh, x, w)
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(first, pol.gated_ffn_grad(dh, x, w)))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("V", [20, 60, 120, 256, 257, 512, 513, 1024])
@pytest.mark.parametrize("top", [1, 2, 7, 20, 32])
def test_alternatives_of_rows_in_registers(pol, V, top, dtype):
    """Many to choose from, ties that fill a list, few entries left, none left, infinities and NaN among the rest."""
    x, tok, mask, _, _ = logp.make(19, V, dtype, V + top)
    top = min(top, V)
    x[0] = 1.5
    x[1] = x[1].round().clamp(-1, 1)
    x[2] = torch.where(torch.arange(V, device="cuda") % 2 == 0, 0.0, -0.0).to(dtype)
    x[3, -min(V, 70):] = 20.0
    x[4] = torch.finfo(dtype).min
    x[5] = float("-inf")
    mask[6] = 0
    mask[7] = 0
    mask[7, [0, V // 2, V - 1]] = 1
    x[8, 1:] = float("-inf")
    logp.check(pol, x, tok, mask, None, None, top, f"{top} of {V} masked")
    logp.check(pol, x, tok, None, None, None, top, f"{top} of {V}")
    x[9, V // 3], x[9, V // 2], x[10, 3], x[11, 5] = float("nan"), float("nan"), float("inf"), -float("nan")
    got = pol.log_probs(x, tok, top=top)["top_index"].cpu()
    assert torch.equal(got, top_of(x.cpu().double(), x.cpu() != float("-inf"), top))
