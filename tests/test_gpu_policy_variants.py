"""The policy operators at the sizes and layouts between which they change their way, against the definitions in 64 bits:
the bounds are those of the operators' own tests, whose `check` functions derive them."""
from __future__ import annotations

import threading

import pytest

torch = pytest.importorskip("torch")

from tests import test_gpu_policy_ffn as ffn  # noqa: E402
from tests import test_gpu_policy_logp as logp  # noqa: E402
from tests import test_gpu_policy_norm as norm  # noqa: E402
from tests import test_gpu_policy_scan as scan  # noqa: E402
from tests.policy_ref import BF16, F16, F32  # noqa: E402

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
