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

AV_F32, AV_BF16, AV_F16 = 0, 1, 2
AV_SILU, AV_GELU = 0, 1
MAX_TOP = 32
_F32, _U8 = torch.float32, torch.uint8
_TYPES = {_F32: AV_F32, torch.bfloat16: AV_BF16, torch.float16: AV_F16}
_ACTS = {"silu": AV_SILU, "gelu": AV_GELU}
_TOKENS = {_U8: 1, torch.int32: 4, torch.int64: 8}
_empty, _empty_like = torch.empty, torch.empty_like
# The current stream's handle by device index: 0.1 us, where making a Stream object takes 2.9.  On small
# inputs a call's time is the host's: what follows keeps to few tensor operations.
_current = torch._C._cuda_getCurrentRawStream


def _tensors(x):
    if isinstance(x, torch.Tensor):
        yield x
    elif isinstance(x, dict):
        for v in x.values():
            yield from _tensors(v)
    elif isinstance(x, (tuple, list)):
        for v in x:
            yield from _tensors(v)


def _on(stream, call, *args):
    """call(*args) whole on another stream."""
    given = list(_tensors(args))
    if not given or not given[0].is_cuda:
        raise ValueError("expected CUDA tensors")
    device = given[0].device
    cur = torch.cuda.current_stream(device)
    handle = _stream(stream)
    if handle == 1:  # the runtime's other name of the legacy default stream
        handle = 0
    if handle == cur.cuda_stream:
        return call(*args)
    on = torch.cuda.ExternalStream(handle, device)
    with torch.cuda.stream(on):
        out = call(*args)
    for x in given:
        x.record_stream(on)
    for x in _tensors(out):
        x.record_stream(cur)
    return out


def _check(fn, rc):
    if rc:
        raise AvError(fn, rc, av_strerror(rc))


def _type(name, x):
    """The library's number of a CUDA tensor's type."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError(f"{name}: expected a CUDA tensor")
    dtype = _TYPES.get(x.dtype)
    if dtype is None:
        raise ValueError(f"{name}: expected float32, bfloat16 or float16, got {x.dtype}")
    return dtype


def _like(name, x, ref, dtype=None, shape=None):
    """x is a tensor on ref's device, of that type and shape."""
    if not isinstance(x, torch.Tensor) or x.device != ref.device:
        raise ValueError(f"{name}: expected a tensor on {ref.device}")
    if dtype is not None and x.dtype != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {x.dtype}")
    if shape is not None and x.shape != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(x.shape)}")


def _dense(name, x, ref, dtype, shape):
    """Pointer of a contiguous tensor of that type and shape (None: a null pointer)."""
    if x is None:
        return None
    _like(name, x, ref, dtype, shape)
    if not x.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor")
    return x.data_ptr()


def _rows(name, x):
    """(rows, n, row stride) of x [..., n] as evenly spaced rows."""
    if x.dim() != 2:
        if x.dim() < 1:
            raise ValueError(f"{name}: expected at least 1 axis")
        try:
            x = x.view(-1, x.shape[-1]) if x.numel() else x.new_empty(x[..., :1].numel(), x.shape[-1])
        except RuntimeError:
            raise ValueError(f"{name}: the rows are not evenly spaced") from None
    rows, n = x.shape
    stride, inner = x.stride()
    if inner != 1 and n > 1:
        raise ValueError(f"{name}: the last axis is not contiguous")
    return rows, n, stride


def _seq(name, x):
    """Strides of a [T, B, D] tensor's steps and sequences."""
    t, b, inner = x.stride()
    if inner != 1 and x.shape[2] > 1:
        raise ValueError(f"{name}: the last axis is not contiguous")
    return t, b


@functools.lru_cache(maxsize=256)
def _norm_work(rows, n):
    need = ctypes.c_int64()
    _check("av_layer_norm_work", load().av_layer_norm_work(rows, n, ctypes.byref(need)))
    return need.value


@functools.lru_cache(maxsize=256)
def _scan_sizes(T, B, D, dtype):
    states, work = ctypes.c_int64(), ctypes.c_int64()
    _check("av_scan_sizes", load().av_scan_sizes(T, B, D, dtype, ctypes.byref(states), ctypes.byref(work)))
    return states.value, work.value


@functools.lru_cache(maxsize=256)
def _ffn_work(rows, D, H):
    need = ctypes.c_int64()
    _check("av_gated_ffn_work", load().av_gated_ffn_work(rows, D, H, ctypes.byref(need)))
    return need.value


def layer_norm(x, weight=None, bias=None, eps=1e-5, stream=None):
    """Layer norm over the last axis of x [..., n]: (y, mean, rstd), mean and
    rstd float32 [...].  weight, bias: [n], of one type."""
    if stream is not None:
        return _on(stream, layer_norm, x, weight, bias, eps)
    dtype = _type("x", x)
    rows, n, stride = _rows("x", x)
    w = b = None
    pt = dtype
    if weight is not None:
        pt = _type("weight", weight)
        w = _dense("weight", weight, x, None, (n,))
    if bias is not None:
        if weight is None:
            pt = _type("bias", bias)
        b = _dense("bias", bias, x, None if weight is None else weight.dtype, (n,))
    dev, shape = x.device, x.shape
    lead = shape[:-1]
    y = _empty(shape, dtype=x.dtype, device=dev)
    mean = _empty(lead, dtype=_F32, device=dev)
    rstd = _empty_like(mean)
    _check("av_layer_norm", load().av_layer_norm(rows, n, dtype, pt, eps, x.data_ptr(), stride, w, b, y.data_ptr(), n,
                                                 mean.data_ptr(), rstd.data_ptr(), _current(x.get_device())))
    return y, mean, rstd


def layer_norm_grad(dy, x, weight, mean, rstd, stream=None):
    """Gradient of layer_norm from dy: (dx, dweight, dbias); the last two are
    [n] of weight's type, or of float32 without a weight."""
    if stream is not None:
        return _on(stream, layer_norm_grad, dy, x, weight, mean, rstd)
    dtype = _type("x", x)
    rows, n, stride = _rows("x", x)
    _like("dy", dy, x, x.dtype, x.shape)
    pt = AV_F32 if weight is None else _type("weight", weight)
    w = _dense("weight", weight, x, None, (n,))
    lead, dev = x.shape[:-1], x.device
    if mean is None or rstd is None:
        raise ValueError("mean, rstd: expected layer_norm's")
    m, r = _dense("mean", mean, x, _F32, lead), _dense("rstd", rstd, x, _F32, lead)
    need = _norm_work(rows, n)
    dx = _empty(x.shape, dtype=x.dtype, device=dev)
    dw = _empty(n, dtype=_F32 if weight is None else weight.dtype, device=dev)
    db = _empty_like(dw)
    work = _empty(need, dtype=_U8, device=dev)
    _check("av_layer_norm_grad", load().av_layer_norm_grad(
        rows, n, dtype, pt, dy.data_ptr(), _rows("dy", dy)[2], x.data_ptr(), stride, w, m, r, dx.data_ptr(), n,
        dw.data_ptr(), db.data_ptr(), work.data_ptr(), need, _current(x.get_device())))
    return dx, dw, db


def _scan_inputs(gate, value, reset):
    dtype = _type("gate", gate)
    if gate.dim() != 3:
        raise ValueError("gate: expected [T, B, D]")
    _like("value", value, gate, gate.dtype, gate.shape)
    where = (gate.data_ptr(), *_seq("gate", gate), value.data_ptr(), *_seq("value", value))
    if reset is None:
        return dtype, (*where, None, 0, 0)
    _like("reset", reset, gate)
    if reset.dtype == torch.bool:
        reset = reset.view(_U8)
    _like("reset", reset, gate, _U8, gate.shape[:2])
    return dtype, (*where, reset.data_ptr(), *reset.stride())


def scan(gate, value, reset=None, h0=None, save=False, stream=None):
    """The gated linear recurrence over time-first trajectories gate, value
    [T, B, D]: (h [T, B, D], h_last float32 [B, D]); with `save` also what
    scan_grad needs.  reset: uint8 or bool [T, B], not 0 where an episode
    begins (for `Env.step`'s trajectories: the done flags of the step before);
    h0: float32 [B, D], zeros if None.  One step when acting: T = 1."""
    if stream is not None:
        return _on(stream, scan, gate, value, reset, h0, save)
    dtype, where = _scan_inputs(gate, value, reset)
    T, B, D = gate.shape
    kept, need = _scan_sizes(T, B, D, dtype)
    first = _dense("h0", h0, gate, _F32, (B, D))
    dev = gate.device
    h = _empty((T, B, D), dtype=gate.dtype, device=dev)
    last = _empty((B, D), dtype=_F32, device=dev)
    states = _empty(kept, dtype=_F32, device=dev) if save else None
    work = _empty(need, dtype=_U8, device=dev) if need else None
    _check("av_scan", load().av_scan(T, B, D, dtype, *where, first, h.data_ptr(), B * D, D, last.data_ptr(),
                                     states.data_ptr() if save else None, work.data_ptr() if need else None, need,
                                     _current(gate.get_device())))
    return (h, last, states) if save else (h, last)


def scan_grad(dh, gate, value, reset, states, dlast=None, stream=None):
    """Gradient of scan from dh (of h) and dlast (float32 [B, D], of h_last):
    (dgate, dvalue, dh0 float32 [B, D])."""
    if stream is not None:
        return _on(stream, scan_grad, dh, gate, value, reset, states, dlast)
    dtype, where = _scan_inputs(gate, value, reset)
    T, B, D = gate.shape
    kept, need = _scan_sizes(T, B, D, dtype)
    _like("dh", dh, gate, gate.dtype, gate.shape)
    if states is None:
        raise ValueError("states: expected what scan kept")
    state, last = _dense("states", states, gate, _F32, (kept,)), _dense("dlast", dlast, gate, _F32, (B, D))
    dev = gate.device
    dgate = _empty((T, B, D), dtype=gate.dtype, device=dev)
    dvalue = _empty_like(dgate)
    dh0 = _empty((B, D), dtype=_F32, device=dev)
    work = _empty(need, dtype=_U8, device=dev) if need else None
    _check("av_scan_grad", load().av_scan_grad(
        T, B, D, dtype, dh.data_ptr(), *_seq("dh", dh), *where, state, last, dgate.data_ptr(), B * D, D,
        dvalue.data_ptr(), B * D, D, dh0.data_ptr(), work.data_ptr() if need else None, need,
        _current(gate.get_device())))
    return dgate, dvalue, dh0


def _logp_inputs(logits, tokens, mask):
    dtype = _type("logits", logits)
    rows, V, stride = _rows("logits", logits)
    _like("tokens", tokens, logits, None, logits.shape[:-1])
    size = _TOKENS.get(tokens.dtype)
    if size is None:
        raise ValueError("tokens: expected uint8, int32 or int64")
    if not tokens.is_contiguous():
        raise ValueError("tokens: expected a contiguous tensor")
    if mask is None:
        return rows, V, (rows, V, dtype, logits.data_ptr(), stride, tokens.data_ptr(), size, None, 0)
    _like("mask", mask, logits)
    if mask.dtype == torch.bool:
        mask = mask.view(_U8)
    _like("mask", mask, logits, _U8)
    if mask.shape == logits.shape:
        apart = _rows("mask", mask)[2]
    elif mask.shape == (V,) and mask.is_contiguous():
        apart = 0
    else:
        raise ValueError(f"mask: expected shape {tuple(logits.shape)} or ({V},)")
    return rows, V, (rows, V, dtype, logits.data_ptr(), stride, tokens.data_ptr(), size, mask.data_ptr(), apart)


def log_probs(logits, tokens, mask=None, top=0, stream=None):
    """Log probabilities of `tokens` [...] under logits [..., V]: dict of
    float32 logp, entropy, peak, logz [...] (the largest logit and the log of the
    sum of exponentials below it) and, with `top`, top_logp float32 and top_index
    int32 [..., top].  tokens: uint8 (`Env.step`'s actions), int32 or
    int64; one outside 0..V-1 has logp 0 and no gradient.  mask: uint8 or bool
    [..., V] or [V], 0 where an entry is not there."""
    if stream is not None:
        return _on(stream, log_probs, logits, tokens, mask, top)
    rows, V, where = _logp_inputs(logits, tokens, mask)
    if not 0 <= top <= min(V, MAX_TOP):
        raise ValueError(f"top: expected 0..{min(V, MAX_TOP)}")
    lead, dev = logits.shape[:-1], logits.device
    logp = _empty(lead, dtype=_F32, device=dev)
    entropy, peak, logz = _empty_like(logp), _empty_like(logp), _empty_like(logp)
    out = {"logp": logp, "entropy": entropy, "peak": peak, "logz": logz}
    values = index = None
    if top:
        out["top_logp"] = best = _empty((*lead, top), dtype=_F32, device=dev)
        out["top_index"] = which = _empty((*lead, top), dtype=torch.int32, device=dev)
        values, index = best.data_ptr(), which.data_ptr()
    _check("av_log_probs", load().av_log_probs(*where, top, logp.data_ptr(), entropy.data_ptr(), peak.data_ptr(),
                                               logz.data_ptr(), values, index, _current(logits.get_device())))
    return out


def log_probs_grad(dlogp, dentropy, logits, tokens, out, mask=None, stream=None):
    """Gradient with respect to logits, from those of logp and entropy (float32
    [...], each may be None) and what log_probs returned."""
    if stream is not None:
        return _on(stream, log_probs_grad, dlogp, dentropy, logits, tokens, out, mask)
    rows, V, where = _logp_inputs(logits, tokens, mask)
    lead = logits.shape[:-1]
    peak, logz = out["peak"], out["logz"]
    if peak is None or logz is None:
        raise ValueError("out: expected what log_probs returned")
    dl, de = _dense("dlogp", dlogp, logits, _F32, lead), _dense("dentropy", dentropy, logits, _F32, lead)
    pk, lz = _dense("peak", peak, logits, _F32, lead), _dense("logz", logz, logits, _F32, lead)
    en = _dense("entropy", out["entropy"], logits, _F32, lead)
    dx = _empty(logits.shape, dtype=logits.dtype, device=logits.device)
    _check("av_log_probs_grad", load().av_log_probs_grad(*where, dl, de, pk, lz, en, dx.data_ptr(), V,
                                                         _current(logits.get_device())))
    return dx


def _ffn_inputs(x, w, act):
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


def gated_ffn(x, w, act="silu", stream=None):
    """h [..., H] = act(x w[0]^T) * (x w[1]^T) for x [..., D], w [2, H, D], of
    one type, bfloat16 or float16; act "silu" or "gelu" (tanh form)."""
    if stream is not None:
        return _on(stream, gated_ffn, x, w, act)
    rows, D, H, dtype, a, stride = _ffn_inputs(x, w, act)
    h = _empty((*x.shape[:-1], H), dtype=x.dtype, device=x.device)
    _check("av_gated_ffn", load().av_gated_ffn(rows, D, H, dtype, a, x.data_ptr(), stride, w.data_ptr(), h.data_ptr(),
                                               H, _current(x.get_device())))
    return h


def gated_ffn_grad(dh, x, w, act="silu", stream=None):
    """Gradient of gated_ffn from dh [..., H]: (dx, dw), of x's and w's shapes."""
    if stream is not None:
        return _on(stream, gated_ffn_grad, dh, x, w, act)
    rows, D, H, dtype, a, stride = _ffn_inputs(x, w, act)
    _like("dh", dh, x, x.dtype, (*x.shape[:-1], H))
    need = _ffn_work(rows, D, H)
    dev = x.device
    dx = _empty(x.shape, dtype=x.dtype, device=dev)
    dw = _empty_like(w)
    work = _empty(need, dtype=_U8, device=dev)
    _check("av_gated_ffn_grad", load().av_gated_ffn_grad(rows, D, H, dtype, a, dh.data_ptr(), _rows("dh", dh)[2],
                                                         x.data_ptr(), stride, w.data_ptr(), dx.data_ptr(), D,
                                                         dw.data_ptr(), work.data_ptr(), need,
                                                         _current(x.get_device())))
    return dx, dw
