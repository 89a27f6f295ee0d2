"""The policy operators at their edges: NaN among the alternatives of long rows, a state that is written where it was
read, calls from two threads, rows of 2^31 - 1 values, arguments
that require gradients, gates of exactly zero."""
from __future__ import annotations

import ctypes
import math
import threading
import warnings

import pytest

torch = pytest.importorskip("torch")

from tests import test_gpu_policy_logp as logp  # noqa: E402
from tests import test_gpu_policy_norm as norm  # noqa: E402
from tests import test_gpu_policy_scan as scan  # noqa: E402
from tests.policy_ref import BF16, F32, close, top_of  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pol():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2407_04221_gb300 import policy
    return policy


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [6, 640])  # by blocks of 512 threads, and of 128
@pytest.mark.parametrize("V", [1025, 1500, 5001])
def test_nan_at_the_first_entry_of_a_long_row(pol, V, rows, dtype):
    """NaN comes before all, the lowest index first: also index 0, alone, with others, and where all are."""
    x, tok, mask, _, _ = logp.make(rows, V, dtype, V)
    x[0, 0] = math.nan
    x[1, [0, V // 2, V - 1]] = math.nan
    x[2] = math.nan
    x[3, [0, 5]] = math.nan
    x[4, 0], x[4, 1] = -math.nan, math.inf
    mask[:] = 1
    mask[3, 0] = 0
    for m in (None, mask):
        there = torch.ones(5, V, dtype=torch.bool) if m is None else m[:5].cpu() != 0
        got = pol.log_probs(x, tok, mask=m, top=7)["top_index"][:5].cpu()
        assert torch.equal(got, top_of(x[:5].cpu().double(), there, 7))


@pytest.mark.parametrize("T,B,D,dtype", [(512, 1, 256, BF16), (5000, 1, 64, F32), (700, 3, 65, BF16), (20, 3, 64, F32),
                                         (6, 64, 64, BF16), (1, 3, 64, F32)])
def test_state_in_its_place(pol, T, B, D, dtype):
    """h_last may be h0 itself, and dh0 dlast: what C callers that step on do.  Long sequences are cut into segments, all
    of which begin from that state; other work on the GPU makes some of them begin late."""
    import paper_2407_04221_gb300 as av
    L = av.load()
    g, v, reset, h0, dh, dlast = scan.make(T, B, D, dtype, 0.001, T, shift=4.0)
    want_h, want_last, states = pol.scan(g, v, reset, h0, save=True)
    want = pol.scan_grad(dh, g, v, reset, states, dlast=dlast)
    kind = {F32: 0, BF16: 1}[dtype]
    n_states, n_work = ctypes.c_int64(), ctypes.c_int64()
    assert L.av_scan_sizes(T, B, D, kind, ctypes.byref(n_states), ctypes.byref(n_work)) == 0
    work = torch.empty(max(n_work.value, 16), dtype=torch.uint8, device="cuda")
    h, dg, dv, kept = torch.empty_like(g), torch.empty_like(g), torch.empty_like(g), torch.empty_like(states)
    busy, side = torch.randn(4096, 4096, device="cuda"), torch.cuda.Stream()
    st, t, b = torch.cuda.current_stream().cuda_stream, B * D, D
    for k in range(20):
        state, flow = h0.clone(), dlast.clone()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            busy @ busy
        args = [g.data_ptr(), t, b, v.data_ptr(), t, b, reset.data_ptr(), B, 1]
        assert L.av_scan(T, B, D, kind, *args, state.data_ptr(), h.data_ptr(), t, b, state.data_ptr(), kept.data_ptr(),
                         work.data_ptr(), n_work.value, st) == 0
        assert L.av_scan_grad(T, B, D, kind, dh.data_ptr(), t, b, *args, kept.data_ptr(), flow.data_ptr(), dg.data_ptr(),
                              t, b, dv.data_ptr(), t, b, flow.data_ptr(), work.data_ptr(), n_work.value, st) == 0
        for got, right in zip((h, state, kept, dg, dv, flow), (want_h, want_last, states, *want)):
            assert torch.equal(got, right), (k, T)


@pytest.mark.parametrize("T", [4, 1000, 20000])
@pytest.mark.parametrize("B,D", [(0, 256), (4, 0)])
def test_scan_of_an_empty_batch(pol, T, B, D):
    g, v, reset, h0, dh, dlast = scan.make(T, B, D, BF16, 0.1, T)
    h, last, states = pol.scan(g, v, reset, h0, save=True)
    assert h.shape == (T, B, D) and last.shape == (B, D) and states.numel() == 0
    dg, dv, dh0 = pol.scan_grad(dh, g, v, reset, states, dlast=dlast)
    assert dg.shape == dv.shape == (T, B, D) and dh0.shape == (B, D)


@pytest.mark.parametrize("gradient", [False, True])
def test_rows_of_two_lengths_from_two_threads(pol, gradient):
    """Two threads with rows that take one kernel and different amounts of shared memory."""
    wrong = []

    def work(n):
        try:
            x, dy, w, b = norm.make(64, n, BF16, F32, n)
            with torch.cuda.stream(torch.cuda.Stream()):
                _, mean, rstd = pol.layer_norm(x, w, b)
                for _ in range(3000):
                    pol.layer_norm_grad(dy, x, w, mean, rstd) if gradient else pol.layer_norm(x, w, b)
        except Exception as e:  # noqa: BLE001
            wrong.append(e)

    threads = [threading.Thread(target=work, args=(n,)) for n in (1024, 4096)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong


LONGEST = 2**31 - 1


def room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 80 * 2**30:
        pytest.skip("not enough memory")


def test_norm_of_the_longest_row(pol):
    """Ones of alternating signs, one more of +1: mean 2^-31, variance 1, so y is x and xh is x to 2^-17 (eps)."""
    room()
    x = torch.ones(1, LONGEST, dtype=BF16, device="cuda")
    x[0, 1::2] = -1
    y, mean, rstd = pol.layer_norm(x)
    assert torch.equal(y, x) and abs(float(mean)) < 1e-6 and abs(float(rstd) - 1) < 1e-5
    del y
    dx, dw, db = pol.layer_norm_grad(x, x, None, mean, rstd)
    assert float(dx.abs().max()) < 1e-4  # (what is left of d - xh mean(d xh))
    assert float((dw - 1).abs_().max()) < 1e-4
    assert float(db[0]) == float(db[-1]) == 1 and float(db[1]) == -1 and float(db.abs_().min()) == 1
    del x, dx, dw, db
    torch.cuda.empty_cache()


@pytest.mark.parametrize("start", [0, 1])
def test_log_probs_of_the_longest_row(pol, start):
    """Zeros and a last entry of 20, its token: sums of 2^21 equal terms a thread are exact to 2^-24."""
    room()
    x = torch.zeros(LONGEST + start, dtype=BF16, device="cuda")[None, start:]
    x[0, -1] = 20
    tok = torch.tensor([LONGEST - 1], device="cuda")
    out = pol.log_probs(x, tok, top=2)
    rest = (LONGEST - 1) * math.exp(-20)
    assert out["top_index"].tolist() == [[LONGEST - 1, 0]] and float(out["peak"]) == 20
    assert abs(float(out["logz"]) - math.log1p(rest)) < 1e-4 and abs(float(out["logp"]) + math.log1p(rest)) < 1e-4
    dx = pol.log_probs_grad(torch.ones(1, device="cuda"), None, x, tok, out)
    p = math.exp(-20) / (1 + rest)
    assert abs(float(dx[0, -1]) / (rest / (1 + rest)) - 1) < 2**-8 + 1e-4
    assert abs(float(dx[0, :-1].min()) / -p - 1) < 2**-8 + 1e-4 and abs(float(dx[0, :-1].max()) / -p - 1) < 2**-8 + 1e-4
    del x, dx
    torch.cuda.empty_cache()


def test_detached_results_are_said(pol):
    """Nothing is recorded by autograd: a call that it would have recorded warns, any other does not."""
    x, dy, w, b = norm.make(8, 64, BF16, F32, 1)
    tok = torch.zeros(8, dtype=torch.int64, device="cuda")
    wants, ffn_w = x.clone().requires_grad_(), torch.zeros(2, 8, 64, dtype=BF16, device="cuda", requires_grad=True)
    calls = [lambda: pol.layer_norm(x, torch.nn.Parameter(w), b), lambda: pol.layer_norm(wants), lambda: pol.log_probs(wants, tok),
             lambda: pol.scan(x[None], wants[None]), lambda: pol.gated_ffn(x, ffn_w),
             lambda: pol.layer_norm(wants, stream=torch.cuda.current_stream())]
    for call in calls:
        with pytest.warns(UserWarning, match="detached"):
            got = call()
        assert not any(t.requires_grad for t in (got.values() if isinstance(got, dict) else got))
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        with torch.no_grad():
            for call in calls:
                call()
        pol.layer_norm(x, w, b)
        pol.layer_norm(wants.detach())

        class Norm(torch.autograd.Function):
            @staticmethod
            def forward(ctx, x):
                y, mean, rstd = pol.layer_norm(x)
                ctx.save_for_backward(x, mean, rstd)
                return y

            @staticmethod
            def backward(ctx, dy):
                x, mean, rstd = ctx.saved_tensors
                return pol.layer_norm_grad(dy, x, None, mean, rstd)[0]

        Norm.apply(wants).backward(dy)
        assert torch.isfinite(wants.grad).all()
        with pytest.raises(UserWarning):
            calls[1]()


@pytest.mark.parametrize("T,B,D,dtype", [(3, 80, 64, F32), (200, 2, 40, BF16), (3000, 1, 33, F32)])
def test_gates_of_zero(pol, T, B, D, dtype):
    """sigmoid(0) = 1/2 with a slope of 1/4: h_t = (h_{t-1} + v_t) / 2, dg_t = l_t (h_{t-1} - v_t) / 4, step by step in 64
    bits; each of these operations is off by at most e of magnitudes below 8 in the kernel, and halves what was before."""
    g, v, _, h0, dh, dlast = scan.make(T, B, D, dtype, None, T)
    g.zero_()
    h, last, states = pol.scan(g, v, None, h0, save=True)
    dg, dv, dh0 = pol.scan_grad(dh, g, v, None, states, dlast=dlast)
    before, state = [], h0.double().cpu()
    for t in range(T):
        before.append(state)
        state = (state + v[t].double().cpu()) / 2
    close(last, state, 8 * 16.0, "last")
    flow = dlast.double().cpu()
    for t in reversed(range(T)):
        flow = flow + dh[t].double().cpu()
        close(dv[t], flow / 2, 8 * 16.0, f"dv {t}")
        close(dg[t], flow * (before[t] - v[t].double().cpu()) / 4, 64 * 16.0, f"dg {t}")
        flow = flow / 2
    close(dh0, flow, 8 * 16.0, "dh0")
