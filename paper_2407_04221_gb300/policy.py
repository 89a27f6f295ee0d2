"""The pieces of a recurrent policy (Sec. 3.2, 3.3): layer norm, a gated linear
recurrence over trajectories, the gated feed-forward, and the log probabilities
of the taken actions, each with its gradient.

Argument marshalling only, as in the package itself: the functions make their
outputs (torch, cuda), check what they are given (ValueError) and call the
library's `av_*` function of the same name, whose description in
`include/autoverse.h` has the formulas and limits.  Nothing waits for the GPU.
Arrays are float32, bfloat16 or float16; innermost axes are contiguous, the
others may have any strides, inputs also those of broadcast (expanded) arrays.

A function given a `stream` runs whole on it, as the calls of `Env` do: its
outputs come from that stream's pool, its arguments are marked as used by that
stream and its results as used by the current one.  It waits for nothing: the
caller orders the streams before the call and before using the results.
"""
from __future__ import annotations

import ctypes
import functools

import torch

from . import AvError, _stream, av_strerror, load

# the current stream's handle by device index: 0.1 us, where making a Stream object takes 2.9
_current = torch._C._cuda_getCurrentRawStream

AV_F32, AV_BF16, AV_F16 = 0, 1, 2
AV_SILU, AV_GELU = 0, 1
MAX_TOP = 32
_TYPES = {torch.float32: AV_F32, torch.bfloat16: AV_BF16, torch.float16: AV_F16}
_ACTS = {"silu": AV_SILU, "gelu": AV_GELU}
_TOKENS = {torch.uint8: 1, torch.int32: 4, torch.int64: 8}


def _tensors(x):
    if isinstance(x, torch.Tensor):
        yield x
    elif isinstance(x, dict):
        for v in x.values():
            yield from _tensors(v)
    elif isinstance(x, (tuple, list)):
        for v in x:
            yield from _tensors(v)


def _on_stream(fn):
    @functools.wraps(fn)
    def call(*args, stream=None, **kw):
        if stream is None:
            return fn(*args, **kw)
        given = list(_tensors([args, kw]))
        device = given[0].device if given else None
        if device is None or device.type != "cuda":
            raise ValueError("expected CUDA tensors")
        cur = torch.cuda.current_stream(device)
        handle = _stream(stream)
        if handle == 1:  # the runtime's other name of the legacy default stream
            handle = 0
        if handle == cur.cuda_stream:
            return fn(*args, **kw)
        on = torch.cuda.ExternalStream(handle, device)
        with torch.cuda.stream(on):
            out = fn(*args, **kw)
        for x in given:
            x.record_stream(on)
        for x in _tensors(out):
            x.record_stream(cur)
        return out
    return call


def _check(fn, rc):
    if rc:
        raise AvError(fn, rc, av_strerror(rc))


def _type(name, x):
    try:
        return _TYPES[x.dtype]
    except (KeyError, AttributeError):
        raise ValueError(f"{name}: expected a float32, bfloat16 or float16 tensor") from None


def _like(name, x, ref, dtype=None, shape=None):
    """x is a tensor on ref's device, of that type and shape."""
    if not isinstance(x, torch.Tensor) or x.device != ref.device:
        raise ValueError(f"{name}: expected a tensor on {ref.device}")
    if dtype is not None and x.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {x.dtype}")
    if shape is not None and tuple(x.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(x.shape)}")


def _dense(name, x, ref, dtype, shape):
    """Pointer of a contiguous tensor of that type and shape (None: a null pointer)."""
    if x is None:
        return None
    _like(name, x, ref, dtype, shape)
    if not x.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor")
    return x.data_ptr()


def _cuda(name, x, ndim):
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError(f"{name}: expected a CUDA tensor")
    if x.dim() < ndim:
        raise ValueError(f"{name}: expected at least {ndim} axes")


def _rows(name, x):
    """(rows, n, row stride) of x [..., n] as evenly spaced rows."""
    if x.dim() != 2:
        try:
            x = x.view(-1, x.shape[-1]) if x.numel() else x.new_empty(x[..., 0].numel(), x.shape[-1])
        except RuntimeError:
            raise ValueError(f"{name}: the rows are not evenly spaced") from None
    rows, n = x.shape
    stride, inner = x.stride()
    if n > 1 and inner != 1:
        raise ValueError(f"{name}: the last axis is not contiguous")
    return rows, n, stride


def _seq(name, x):
    """Strides of a [T, B, D] tensor's steps and sequences."""
    t, b, inner = x.stride()
    if x.shape[2] > 1 and inner != 1:
        raise ValueError(f"{name}: the last axis is not contiguous")
    return t, b


@_on_stream
def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Layer norm over the last axis of x [..., n]: (y, mean, rstd), mean and
    rstd float32 [...].  weight, bias: [n], of one type."""
    _cuda("x", x, 1)
    dtype = _type("x", x)
    rows, n, stride = _rows("x", x)
    param = weight if weight is not None else bias
    pt = dtype if param is None else _type("weight", param)
    w = _dense("weight", weight, x, None, (n,))
    b = _dense("bias", bias, x, None if param is None else param.dtype, (n,))
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    mean = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    _check("av_layer_norm", load().av_layer_norm(rows, n, dtype, pt, eps, x.data_ptr(), stride, w, b, y.data_ptr(), n,
                                                 mean.data_ptr(), rstd.data_ptr(), _current(x.get_device())))
    return y, mean, rstd


@_on_stream
def layer_norm_grad(dy, x, weight, mean, rstd):
    """Gradient of layer_norm from dy: (dx, dweight, dbias); the last two are
    [n] of weight's type, or of float32 without a weight."""
    _cuda("x", x, 1)
    dtype = _type("x", x)
    rows, n, stride = _rows("x", x)
    _like("dy", dy, x, x.dtype, x.shape)
    pt = AV_F32 if weight is None else _type("weight", weight)
    w = _dense("weight", weight, x, None, (n,))
    m, r = (_dense(k, v, x, torch.float32, x.shape[:-1]) for k, v in (("mean", mean), ("rstd", rstd)))
    L = load()
    need = ctypes.c_int64()
    _check("av_layer_norm_work", L.av_layer_norm_work(rows, n, ctypes.byref(need)))
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    dw = torch.empty(n, dtype=torch.float32 if weight is None else weight.dtype, device=x.device)
    db = torch.empty_like(dw)
    work = torch.empty(need.value, dtype=torch.uint8, device=x.device)
    _check("av_layer_norm_grad", L.av_layer_norm_grad(
        rows, n, dtype, pt, dy.data_ptr(), _rows("dy", dy)[2], x.data_ptr(), stride, w, m, r, dx.data_ptr(), n,
        dw.data_ptr(), db.data_ptr(), work.data_ptr(), need.value, _current(x.get_device())))
    return dx, dw, db


def _scan_inputs(gate, value, reset):
    _cuda("gate", gate, 3)
    dtype = _type("gate", gate)
    if gate.dim() != 3:
        raise ValueError("gate: expected [T, B, D]")
    _like("value", value, gate, gate.dtype, gate.shape)
    T, B, D = gate.shape
    where = [gate.data_ptr(), *_seq("gate", gate), value.data_ptr(), *_seq("value", value)]
    if reset is None:
        where += [None, 0, 0]
    else:
        _like("reset", reset, gate)
        if reset.dtype == torch.bool:
            reset = reset.view(torch.uint8)
        _like("reset", reset, gate, torch.uint8, (T, B))
        where += [reset.data_ptr(), *reset.stride()]
    states, work = ctypes.c_int64(), ctypes.c_int64()
    _check("av_scan_sizes", load().av_scan_sizes(T, B, D, dtype, ctypes.byref(states), ctypes.byref(work)))
    return dtype, (T, B, D), where, states.value, work.value


@_on_stream
def scan(gate, value, reset=None, h0=None, save=False):
    """The gated linear recurrence over time-first trajectories gate, value
    [T, B, D]: (h [T, B, D], h_last float32 [B, D]); with `save` also what
    scan_grad needs.  reset: uint8 or bool [T, B], not 0 where an episode
    begins (for `Env.step`'s trajectories: the done flags of the step before);
    h0: float32 [B, D], zeros if None.  One step when acting: T = 1."""
    dtype, (T, B, D), where, kept, need = _scan_inputs(gate, value, reset)
    first = _dense("h0", h0, gate, torch.float32, (B, D))
    dev = gate.device
    h = torch.empty((T, B, D), dtype=gate.dtype, device=dev)
    last = torch.empty((B, D), dtype=torch.float32, device=dev)
    states = torch.empty(kept, dtype=torch.float32, device=dev) if save else None
    work = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _check("av_scan", load().av_scan(T, B, D, dtype, *where, first, h.data_ptr(), B * D, D, last.data_ptr(),
                                     states.data_ptr() if save else None, work.data_ptr() if need else None, need,
                                     _current(gate.get_device())))
    return (h, last, states) if save else (h, last)


@_on_stream
def scan_grad(dh, gate, value, reset, states, dlast=None):
    """Gradient of scan from dh (of h) and dlast (float32 [B, D], of h_last):
    (dgate, dvalue, dh0 float32 [B, D])."""
    dtype, (T, B, D), where, kept, need = _scan_inputs(gate, value, reset)
    _like("dh", dh, gate, gate.dtype, gate.shape)
    state = _dense("states", states, gate, torch.float32, (kept,))
    last = _dense("dlast", dlast, gate, torch.float32, (B, D))
    dev = gate.device
    dgate = torch.empty((T, B, D), dtype=gate.dtype, device=dev)
    dvalue = torch.empty_like(dgate)
    dh0 = torch.empty((B, D), dtype=torch.float32, device=dev)
    work = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _check("av_scan_grad", load().av_scan_grad(
        T, B, D, dtype, dh.data_ptr(), *_seq("dh", dh), *where, state, last, dgate.data_ptr(), B * D, D,
        dvalue.data_ptr(), B * D, D, dh0.data_ptr(), work.data_ptr() if need else None, need,
        _current(gate.get_device())))
    return dgate, dvalue, dh0


def _logp_inputs(logits, tokens, mask):
    _cuda("logits", logits, 1)
    dtype = _type("logits", logits)
    rows, V, stride = _rows("logits", logits)
    _like("tokens", tokens, logits, None, logits.shape[:-1])
    if tokens.dtype not in _TOKENS:
        raise ValueError("tokens: expected uint8, int32 or int64")
    if not tokens.is_contiguous():
        raise ValueError("tokens: expected a contiguous tensor")
    allowed, mask_stride = None, 0
    if mask is not None:
        _like("mask", mask, logits)
        if mask.dtype == torch.bool:
            mask = mask.view(torch.uint8)
        _like("mask", mask, logits, torch.uint8)
        if mask.shape != logits.shape and tuple(mask.shape) != (V,):
            raise ValueError(f"mask: expected shape {tuple(logits.shape)} or ({V},)")
        per_row, _, mask_stride = _rows("mask", mask)
        allowed = mask.data_ptr()
        if mask.dim() == 1 and logits.dim() > 1:
            mask_stride = 0
    return rows, V, (rows, V, dtype, logits.data_ptr(), stride, tokens.data_ptr(), _TOKENS[tokens.dtype], allowed,
                     mask_stride)


@_on_stream
def log_probs(logits, tokens, mask=None, top=0):
    """Log probabilities of `tokens` [...] under logits [..., V]: dict of
    float32 logp, entropy, peak, logz [...] (the largest logit and the log of the
    sum of exponentials below it) and, with `top`, top_logp float32 and top_index
    int32 [..., top].  tokens: uint8 (`Env.step`'s actions), int32 or
    int64; one outside 0..V-1 has logp 0 and no gradient.  mask: uint8 or bool
    [..., V] or [V], 0 where an entry is not there."""
    rows, V, where = _logp_inputs(logits, tokens, mask)
    if not 0 <= top <= min(V, MAX_TOP):
        raise ValueError(f"top: expected 0..{min(V, MAX_TOP)}")
    lead, dev = logits.shape[:-1], logits.device
    out = {k: torch.empty(lead, dtype=torch.float32, device=dev) for k in ("logp", "entropy", "peak", "logz")}
    values = index = None
    if top:
        out["top_logp"] = torch.empty((*lead, top), dtype=torch.float32, device=dev)
        out["top_index"] = torch.empty((*lead, top), dtype=torch.int32, device=dev)
        values, index = out["top_logp"].data_ptr(), out["top_index"].data_ptr()
    _check("av_log_probs", load().av_log_probs(
        *where, top, out["logp"].data_ptr(), out["entropy"].data_ptr(), out["peak"].data_ptr(), out["logz"].data_ptr(),
        values, index, _current(logits.get_device())))
    return out


@_on_stream
def log_probs_grad(dlogp, dentropy, logits, tokens, out, mask=None):
    """Gradient with respect to logits, from those of logp and entropy (float32
    [...], each may be None) and what log_probs returned."""
    rows, V, where = _logp_inputs(logits, tokens, mask)
    lead = logits.shape[:-1]
    dl, de, pk, lz, en = (_dense(k, v, logits, torch.float32, lead) for k, v in
                          (("dlogp", dlogp), ("dentropy", dentropy), ("peak", out["peak"]), ("logz", out["logz"]),
                           ("entropy", out["entropy"])))
    dx = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    _check("av_log_probs_grad", load().av_log_probs_grad(*where, dl, de, pk, lz, en, dx.data_ptr(), V,
                                                         _current(logits.get_device())))
    return dx


def _ffn_inputs(x, w, act):
    _cuda("x", x, 1)
    dtype = _type("x", x)
    if dtype == AV_F32:
        raise ValueError("x: expected bfloat16 or float16")
    if act not in _ACTS:
        raise ValueError(f"act: expected one of {sorted(_ACTS)}")
    rows, D, stride = _rows("x", x)
    _like("w", w, x, x.dtype)
    if w.dim() != 3 or w.shape[0] != 2 or w.shape[2] != D or not w.is_contiguous():
        raise ValueError(f"w: expected a contiguous [2, H, {D}] tensor")
    return rows, D, w.shape[1], dtype, _ACTS[act], stride


@_on_stream
def gated_ffn(x, w, act="silu"):
    """h [..., H] = act(x w[0]^T) * (x w[1]^T) for x [..., D], w [2, H, D], of
    one type, bfloat16 or float16; act "silu" or "gelu" (tanh form)."""
    rows, D, H, dtype, a, stride = _ffn_inputs(x, w, act)
    h = torch.empty((*x.shape[:-1], H), dtype=x.dtype, device=x.device)
    _check("av_gated_ffn", load().av_gated_ffn(rows, D, H, dtype, a, x.data_ptr(), stride, w.data_ptr(), h.data_ptr(),
                                               H, _current(x.get_device())))
    return h


@_on_stream
def gated_ffn_grad(dh, x, w, act="silu"):
    """Gradient of gated_ffn from dh [..., H]: (dx, dw), of x's and w's shapes."""
    rows, D, H, dtype, a, stride = _ffn_inputs(x, w, act)
    _like("dh", dh, x, x.dtype, (*x.shape[:-1], H))
    L = load()
    need = ctypes.c_int64()
    _check("av_gated_ffn_work", L.av_gated_ffn_work(rows, D, H, ctypes.byref(need)))
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    dw = torch.empty_like(w)
    work = torch.empty(need.value, dtype=torch.uint8, device=x.device)
    _check("av_gated_ffn_grad", L.av_gated_ffn_grad(rows, D, H, dtype, a, dh.data_ptr(), _rows("dh", dh)[2],
                                                    x.data_ptr(), stride, w.data_ptr(), dx.data_ptr(), D,
                                                    dw.data_ptr(), work.data_ptr(), need.value,
                                                    _current(x.get_device())))
    return dx, dw
