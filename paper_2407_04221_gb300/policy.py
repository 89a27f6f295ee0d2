"""The pieces of a recurrent policy (Sec. 3.2, 3.3): layer norm, a gated linear
recurrence over trajectories, the gated feed-forward, and the log probabilities
of the taken actions, each with its gradient.

Argument marshalling only, as in the package itself: the functions make their
outputs (torch, cuda), check what they are given (ValueError) and call the
library's `av_*` function of the same name (in `csrc/policy_binding.cpp`), whose description in
`include/autoverse.h` has the formulas and limits.  Nothing waits for the GPU.
Arrays are float32, bfloat16 or float16 (the feed-forward's the latter two) and
their innermost axes contiguous.  The axes before are taken together as rows,
which are evenly spaced: whole arrays, parts of wider rows, every second row, one
row expanded to many, but not two axes transposed.  The recurrence's steps and
sequences have strides of their own, whatever they are.  The feed-forward takes
rows that are apart, on 16 bytes and of a multiple of eight values, and its
AvError (AV_EINVAL) says when they are not.

Nothing is recorded by autograd: results are detached, and a call whose
arguments require gradients warns of it where gradients are enabled.  Each
gradient has a function of its own; `examples/recurrent_policy.py` makes
`torch.autograd.Function`s of them.

A function given a `stream` runs whole on it, as the calls of `Env` do: its
outputs come from that stream's pool, its arguments are marked as used by that
stream and its results as used by the current one.  It waits for nothing: the
caller orders the streams before the call and before using the results.
"""
from __future__ import annotations

import importlib
import os

import torch

from . import AvError, _stream, load

AV_F32, AV_BF16, AV_F16 = 0, 1, 2
AV_SILU, AV_GELU = 0, 1
MAX_TOP = 32
_native = None


def _load():
    """The compiled binding; raises if it is missing (no fallback)."""
    global _native
    load()
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_policy.so")
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`")
    native = importlib.import_module("._policy", __package__)
    native.set_error(AvError)
    _native = native
    return native


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


def layer_norm(x, weight=None, bias=None, eps=1e-5, stream=None):
    """Layer norm over the last axis of x [..., n]: (y, mean, rstd), mean and
    rstd float32 [...].  weight, bias: [n], of one type."""
    if stream is not None:
        return _on(stream, layer_norm, x, weight, bias, eps)
    return (_native or _load()).layer_norm(x, weight, bias, eps)


def layer_norm_grad(dy, x, weight, mean, rstd, stream=None):
    """Gradient of layer_norm from dy: (dx, dweight, dbias); the last two are
    [n] of weight's type, or of float32 without a weight."""
    if stream is not None:
        return _on(stream, layer_norm_grad, dy, x, weight, mean, rstd)
    return (_native or _load()).layer_norm_grad(dy, x, weight, mean, rstd)


def scan(gate, value, reset=None, h0=None, save=False, stream=None):
    """The gated linear recurrence over time-first trajectories gate, value
    [T, B, D]: (h [T, B, D], h_last float32 [B, D]); with `save` also what
    scan_grad needs.  reset: uint8 or bool [T, B], not 0 where an episode
    begins (for `Env.step`'s trajectories: the done flags of the step before);
    h0: float32 [B, D], zeros if None.  One step when acting: T = 1."""
    if stream is not None:
        return _on(stream, scan, gate, value, reset, h0, save)
    return (_native or _load()).scan(gate, value, reset, h0, save)


def scan_grad(dh, gate, value, reset, states, dlast=None, stream=None):
    """Gradient of scan from dh (of h) and dlast (float32 [B, D], of h_last):
    (dgate, dvalue, dh0 float32 [B, D])."""
    if stream is not None:
        return _on(stream, scan_grad, dh, gate, value, reset, states, dlast)
    return (_native or _load()).scan_grad(dh, gate, value, reset, states, dlast)


def log_probs(logits, tokens, mask=None, top=0, stream=None):
    """Log probabilities of `tokens` [...] under logits [..., V]: dict of
    float32 logp, entropy, peak, logz [...] (the largest logit and the log of the
    sum of exponentials below it) and, with `top`, top_logp float32 and top_index
    int32 [..., top].  tokens: uint8 (`Env.step`'s actions), int32 or
    int64; one outside 0..V-1 has logp 0 and no gradient.  mask: uint8 or bool
    [..., V] or [V], 0 where an entry is not there."""
    if stream is not None:
        return _on(stream, log_probs, logits, tokens, mask, top)
    return (_native or _load()).log_probs(logits, tokens, mask, top)


def log_probs_grad(dlogp, dentropy, logits, tokens, out, mask=None, stream=None):
    """Gradient with respect to logits, from those of logp and entropy (float32
    [...], each may be None) and what log_probs returned."""
    if stream is not None:
        return _on(stream, log_probs_grad, dlogp, dentropy, logits, tokens, out, mask)
    return (_native or _load()).log_probs_grad(dlogp, dentropy, logits, tokens, out["peak"], out["logz"], out["entropy"], mask)


def gated_ffn(x, w, act="silu", stream=None):
    """h [..., H] = act(x w[0]^T) * (x w[1]^T) for x [..., D], w [2, H, D], of
    one type, bfloat16 or float16; act "silu" or "gelu" (tanh form)."""
    if stream is not None:
        return _on(stream, gated_ffn, x, w, act)
    return (_native or _load()).gated_ffn(x, w, act)


def gated_ffn_grad(dh, x, w, act="silu", stream=None):
    """Gradient of gated_ffn from dh [..., H]: (dx, dw), of x's and w's shapes."""
    if stream is not None:
        return _on(stream, gated_ffn_grad, dh, x, w, act)
    return (_native or _load()).gated_ffn_grad(dh, x, w, act)
