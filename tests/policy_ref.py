"""The policy operators from their definitions, in 64 bits on the CPU, with gradients by torch's autograd, and the
comparison of a kernel's output with them.

Tolerances are error bounds.  With u the unit roundoff of the output's type and e = 2^-24 that of the sums,

    |got - want| <= 1.01 u |want| + e scale + smallest,

where scale bounds what 32-bit evaluation may add (each test states its own) and smallest is half the output type's
smallest subnormal step."""
from __future__ import annotations

import math

import torch

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
ROUNDOFF = {F32: 2.0**-24, BF16: 2.0**-8, F16: 2.0**-11}
SMALLEST = {F32: 2.0**-126, BF16: 2.0**-126, F16: 2.0**-25}
E = 2.0**-24


def close(got, want, scale, what="", rounding=None):
    """`rounding`: a further absolute allowance, for values rounded on the way."""
    u = ROUNDOFF[got.dtype]
    got, want = got.detach().cpu().double(), want.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(got), inf) and torch.equal(got[inf], want[inf]), what
    fine = torch.isfinite(want)
    allowed = 1.01 * u * want.abs() + E * torch.as_tensor(scale, dtype=torch.float64) + SMALLEST[
        {2.0**-24: F32, 2.0**-8: BF16, 2.0**-11: F16}[u]]
    if rounding is not None:
        allowed = allowed + rounding
    off = ((got - want).abs() - allowed).expand(want.shape)[fine]
    if off.numel():
        k = off.argmax()
        assert off[k] <= 0, (what, "off by", float(off[k]), "over the bound at", int(k), float(got[fine][k]),
                             float(want[fine][k]))


def d(x):
    return None if x is None else x.detach().cpu().double()


def layer_norm(x, w, b, eps):
    m = x.mean(-1, keepdim=True)
    var = ((x - m) ** 2).mean(-1, keepdim=True)
    y = (x - m) / (var + eps).sqrt()
    y = y if w is None else y * w
    return y if b is None else y + b


def scan(g, v, reset, h0):
    """Step by step; a reset forgets the state, whatever it is."""
    T = g.shape[0]
    # the gate and its complement, each from the smaller of the two: autograd takes a sigmoid's slope from the
    # sigmoid itself, which would cancel where it is near one
    low, rest = torch.sigmoid(-g.abs()), 1 - torch.sigmoid(-g.abs())
    a, z = torch.where(g > 0, rest, low), torch.where(g > 0, low, rest)
    state = torch.zeros(g.shape[1:], dtype=torch.float64) if h0 is None else h0
    out = []
    for t in range(T):
        if reset is not None:
            state = torch.where((reset[t] != 0)[:, None], torch.zeros_like(state), state)
        state = a[t] * state + z[t] * v[t]
        out.append(state)
    return (torch.stack(out) if out else torch.empty(g.shape, dtype=torch.float64)), state


def log_probs(x, tokens, mask):
    """(logp, entropy, peak, logz, log p, present) of rows x [N, V]; rows with nothing left as the operator defines them."""
    present = torch.ones_like(x, dtype=torch.bool) if mask is None else (mask != 0).expand(x.shape)
    x = torch.where(present, x, torch.full_like(x, -math.inf))
    present = present & (x.detach() != -math.inf)
    some = present.any(1)
    safe = torch.where(some[:, None], x, torch.zeros_like(x))
    peak = safe.detach().amax(1)
    low = safe - peak[:, None]  # (before the logarithm is added: 64 bits would not hold both)
    logz = torch.logsumexp(low, 1)
    logs = torch.where(present, low - logz[:, None], torch.full_like(x, -math.inf))
    none = torch.full_like(peak, -math.inf)
    peak, logz = torch.where(some, peak, none), torch.where(some, logz, none)
    finite = torch.where(present, logs, torch.zeros_like(logs))
    entropy = -(torch.where(present, finite.exp(), torch.zeros_like(logs)) * finite).sum(1)
    given = (tokens >= 0) & (tokens < x.shape[1])
    at = torch.where(given, tokens, torch.zeros_like(tokens)).long()
    logp = torch.where(given, logs.gather(1, at[:, None])[:, 0], torch.zeros_like(entropy))
    return logp, entropy, peak, logz, logs, present


def top_of(x, present, k):
    """Indices of the k largest entries present, NaN first, the lowest index among equals; -1 where none is left."""
    out = torch.full((x.shape[0], k), -1, dtype=torch.int32)
    for r in range(x.shape[0]):
        at = [j for j in range(x.shape[1]) if present[r, j]]
        row = x[r].tolist()
        at.sort(key=lambda j: (0 if math.isnan(row[j]) else 1, 0.0 if math.isnan(row[j]) else -row[j], j))
        for i, j in enumerate(at[:k]):
            out[r, i] = j
    return out


def activate(g, act):
    if act == "silu":
        return g * torch.sigmoid(g)
    return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))


def gated_ffn(x, w, act):
    return activate(x @ w[0].t(), act) * (x @ w[1].t())
