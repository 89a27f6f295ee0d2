"""Performance cases of the policy operators: the pieces of a recurrent policy that acts in the environments and
learns from their trajectories, each through the public calls of `paper_2407_04221_gb300.policy`.

  norm   `layer_norm`, and `layer_norm_grad` with the reduction of the weight's and the bias's gradient
  scan   `scan`, the gated linear recurrence over a trajectory with episode ends, and `scan_grad`; one step when acting
  logp   `log_probs` of given tokens with entropy and top alternatives, and `log_probs_grad`
  ffn    `gated_ffn`, both projections, the activation and the product, and `gated_ffn_grad`

`train` cases run the forward and the backward pass.  With `own` false, `run` computes the same from elementary torch
operations in 32 bits, rounded once at the end.  `exact` computes it in 64 bits from the definitions.
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5


def listed():
    return [
        # one environment's features before its policy's next layer: the smallest call, all latency
        dict(name="norm-act-1x256", op="norm", rows=1, n=256, dtype="bf16", params="f32", train=False),
        # a training batch of 512 environments x 128 steps, parameters kept in 32 bits
        dict(name="norm-train-65536x1024", op="norm", rows=65536, n=1024, dtype="bf16", params="f32", train=True),
        # flattened odd observation windows (31 x 31 x 5) in 32 bits, a ragged number of rows
        dict(name="norm-train-odd-5003x4805", op="norm", rows=5003, n=4805, dtype="f32", params="f32", train=True),
        # the acting step of 16,384 environments: one step of the recurrence
        dict(name="scan-act-16384x256", op="scan", T=1, B=16384, D=256, dtype="bf16", resets=0.01, train=False),
        # a rollout's trajectories, time first, episodes of about 200 steps
        dict(name="scan-train-128x1024x256", op="scan", T=128, B=1024, D=256, dtype="bf16", resets=0.005, train=True),
        # one long trace in 32 bits, odd in length and width
        dict(name="scan-train-long-65537x1x1021", op="scan", T=65537, B=1, D=1021, dtype="f32", resets=0.0005,
             train=True),
        # one environment choosing among the five actions
        dict(name="logp-act-1x5", op="logp", rows=1, V=5, dtype="f32", top=5, mask=True, train=False),
        # the policy loss over 16,384 environments x 64 steps, impossible actions masked
        dict(name="logp-train-1048576x5", op="logp", rows=1048576, V=5, dtype="f32", top=1, mask=True, train=True),
        # a world model's loss over cell words of 16 tile channels, odd in rows, unknown cells without a token
        dict(name="logp-train-2047x65536", op="logp", rows=2047, V=65536, dtype="bf16", top=8, mask=False, train=True),
        # four environments' step through a wide block: the weights are the work
        dict(name="ffn-act-4x1024x4096", op="ffn", rows=4, D=1024, H=4096, act="silu", dtype="bf16", train=False),
        # a training batch, the usual ratio of widths
        dict(name="ffn-train-16384x1024x4096", op="ffn", rows=16384, D=1024, H=4096, act="silu", dtype="bf16",
             train=True),
        # ragged rows, widths that are no powers of two
        dict(name="ffn-train-odd-4099x520x1368", op="ffn", rows=4099, D=520, H=1368, act="gelu", dtype="f16",
             train=True),
    ]


def _log(rng, lo, hi):
    while True:
        n = int(round(lo * (hi / lo) ** rng.random()))
        if n != 3072:
            return n


def draw(rng):
    """One more case of the ranges above: any operator, rows from one to about a million, rows' widths of 16 to
    16,384, 2 to 65,536 tokens, 1 to 65,536 steps, feed-forward widths in eights; every type, with and without
    training."""
    op = rng.choice(("norm", "scan", "logp", "ffn"))
    train, dtype = rng.random() < 0.7, rng.choice(("f32", "bf16", "bf16", "f16"))
    if op == "norm":
        n = _log(rng, 16, 16384)
        return dict(op=op, rows=_log(rng, 1, min(1 << 20, (24 << 20) // n)), n=n, dtype=dtype,
                    params="f32" if rng.random() < 0.6 else dtype, train=train)
    if op == "scan":
        T = 1 if rng.random() < 0.2 else _log(rng, 2, 65536)
        D = _log(rng, 16, 2048)
        return dict(op=op, T=T, B=_log(rng, 1, max(1, min(16384, (32 << 20) // (T * D)))), D=D, dtype=dtype,
                    resets=rng.choice((0.0, 0.001, 0.01, 0.1)), train=train)
    if op == "logp":
        V = _log(rng, 2, 65536)
        return dict(op=op, rows=_log(rng, 1, max(1, min(1 << 20, (64 << 20) // V))), V=V, dtype=dtype,
                    top=rng.randint(0, min(V, 20)), mask=rng.random() < 0.3, train=train)
    D, H = 8 * _log(rng, 8, 256), 8 * _log(rng, 8, 768)
    while 3072 in (D, H):
        D, H = 8 * _log(rng, 8, 256), 8 * _log(rng, 8, 768)
    return dict(op=op, rows=_log(rng, 1, min(32768, (64 << 30) // (D * H))), D=D, H=H,
                act=rng.choice(("silu", "gelu")), dtype=rng.choice(("bf16", "f16")), train=train)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=dt):
        return (torch.randn(*shape, generator=gen, device=DEVICE) * scale).to(dtype)

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device=DEVICE)

    s = dict(case=case)
    if case["op"] == "norm":
        rows, n, pt = case["rows"], case["n"], DTYPES[case["params"]]
        s["x"] = normal(rows, n) + normal(rows, 1, scale=0.5)  # rows with means of their own
        s["weight"] = (1 + normal(n, scale=0.1, dtype=torch.float32)).to(pt)
        s["bias"] = normal(n, scale=0.1, dtype=pt)
        s["dy"] = normal(rows, n)
    elif case["op"] == "scan":
        T, B, D = case["T"], case["B"], case["D"]
        s["gate"] = normal(T, B, D, scale=1.5) + 2.0  # gates near 0.88: a memory of some ten to a hundred steps
        s["value"] = normal(T, B, D)
        s["reset"] = (uniform(T, B) < case["resets"]).to(torch.uint8)
        s["h0"] = normal(B, D, scale=0.5, dtype=torch.float32)
        if case["train"]:
            s["dh"] = normal(T, B, D)
            s["dlast"] = normal(B, D, dtype=torch.float32)
    elif case["op"] == "logp":
        rows, V = case["rows"], case["V"]
        s["logits"] = normal(rows, V, scale=2.0)
        s["tokens"] = torch.randint(0, V, (rows,), generator=gen, device=DEVICE)
        if not case["mask"]:
            s["tokens"][uniform(rows) < 0.05] = -1  # positions without a token
        # now and then a row of few possible tokens has none left
        s["mask"] = (uniform(rows, V) < 0.8).to(torch.uint8) if case["mask"] else None
        s["dlogp"] = normal(rows, dtype=torch.float32)
        s["dentropy"] = normal(rows, scale=0.01, dtype=torch.float32)
    else:
        rows, D, H = case["rows"], case["D"], case["H"]
        s["x"] = normal(rows, D)
        s["w"] = normal(2, H, D, scale=1.0 / math.sqrt(D))
        s["dh"] = normal(rows, H)
    return s


def run(s):
    op = s["case"]["op"]
    if own:
        return {"norm": _own_norm, "scan": _own_scan, "logp": _own_logp, "ffn": _own_ffn}[op](s, s["case"])
    return {"norm": _plain_norm, "scan": _plain_scan, "logp": _plain_logp, "ffn": _plain_ffn}[op](s, s["case"])


# ---------------------------------------------------------------- the framework's calls

def _policy():
    from paper_2407_04221_gb300 import policy
    return policy


def _own_norm(s, case):
    pol = _policy()
    y, mean, rstd = pol.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS)
    if not case["train"]:
        return y
    return (y, *pol.layer_norm_grad(s["dy"], s["x"], s["weight"], mean, rstd))


def _own_scan(s, case):
    pol = _policy()
    if not case["train"]:
        return pol.scan(s["gate"], s["value"], s["reset"], s["h0"])
    h, last, states = pol.scan(s["gate"], s["value"], s["reset"], s["h0"], save=True)
    return (h, last, *pol.scan_grad(s["dh"], s["gate"], s["value"], s["reset"], states, dlast=s["dlast"]))


def _own_logp(s, case):
    pol = _policy()
    out = pol.log_probs(s["logits"], s["tokens"], mask=s["mask"], top=case["top"])
    if not case["train"]:
        return out
    return out, pol.log_probs_grad(s["dlogp"], s["dentropy"], s["logits"], s["tokens"], out, mask=s["mask"])


def _own_ffn(s, case):
    pol = _policy()
    h = pol.gated_ffn(s["x"], s["w"], act=case["act"])
    if not case["train"]:
        return h
    return (h, *pol.gated_ffn_grad(s["dh"], s["x"], s["w"], act=case["act"]))


# ---------------------------------------------------------------- the plain forms

def _plain_norm(s, case):
    x, w, b = s["x"].float(), s["weight"].float(), s["bias"].float()
    xc = x - x.mean(1, keepdim=True)
    rstd = torch.rsqrt((xc * xc).mean(1, keepdim=True) + EPS)
    xh = xc * rstd
    y = (xh * w + b).to(s["x"].dtype)
    if not case["train"]:
        return y
    dy = s["dy"].float()
    d = dy * w
    dx = rstd * (d - d.mean(1, keepdim=True) - xh * (d * xh).mean(1, keepdim=True))
    pt = s["weight"].dtype
    return y, dx.to(s["x"].dtype), (dy * xh).sum(0).to(pt), dy.sum(0).to(pt)


def _recur(c, b):
    """y_t = c_t y_{t-1} + b_t along the first axis, from y_0 = b_0, by doubling: after each round a value stands
    for twice as many steps."""
    step = 1
    while step < b.shape[0]:
        b = torch.cat((b[:step], b[step:] + c[step:] * b[:-step]))
        c = torch.cat((c[:step], c[step:] * c[:-step]))
        step *= 2
    return b


def _plain_scan(s, case):
    dt = s["gate"].dtype
    g, v, h0 = s["gate"].float(), s["value"].float(), s["h0"]
    keep = 1.0 - s["reset"].float()[:, :, None]
    a, z = 1.0 / (1.0 + torch.exp(-g)), 1.0 / (1.0 + torch.exp(g))  # z = 1 - a, without its cancellation
    c, b = a * keep, z * v
    h = _recur(c, torch.cat((b[:1] + c[:1] * h0, b[1:])))
    if not case["train"]:
        return h.to(dt), h[-1]
    dh = s["dh"].float()
    dh = torch.cat((dh[:-1], dh[-1:] + s["dlast"]))
    later = torch.cat((c[1:], torch.zeros_like(c[:1])))
    lam = _recur(later.flip(0), dh.flip(0)).flip(0)
    before = torch.cat((h0[None], h[:-1])) * keep
    return h.to(dt), h[-1], (lam * (before - v) * a * z).to(dt), (lam * z).to(dt), (c[:1] * lam[:1])[0]


def _plain_logp(s, case):
    x, tok = s["logits"].float(), s["tokens"]
    if s["mask"] is not None:
        x = torch.where(s["mask"] != 0, x, torch.tensor(-math.inf, device=x.device))
    top = x.max(1, keepdim=True).values
    some = top > -math.inf  # rows with an entry left
    e = torch.exp(x - torch.where(some, top, torch.zeros_like(top)))
    total = e.sum(1, keepdim=True)
    logz = torch.where(some, torch.log(total), top)
    logs = torch.where(some & (x > -math.inf), (x - top) - logz, torch.full_like(x, -math.inf))
    p = e / torch.where(some, total, torch.ones_like(total))
    entropy = -(p * torch.where(p > 0, logs, torch.zeros_like(p))).sum(1)
    given = (tok >= 0) & (tok < case["V"])
    at = torch.where(given, tok, torch.zeros_like(tok))[:, None]
    out = dict(logp=torch.where(given, logs.gather(1, at)[:, 0], torch.zeros_like(entropy)), entropy=entropy,
               peak=top[:, 0], logz=logz[:, 0])
    if case["top"]:
        best, index = torch.sort(x, dim=1, descending=True, stable=True)
        best, index = best[:, :case["top"]], index[:, :case["top"]]
        there = best > -math.inf
        out["top_logp"] = torch.where(there, (best - top) - logz, best)
        out["top_index"] = torch.where(there, index, torch.full_like(index, -1)).to(torch.int32)
    if not case["train"]:
        return out
    there = (x > -math.inf) & some
    dlogp, dent = torch.where(given, s["dlogp"], torch.zeros_like(s["dlogp"])), s["dentropy"]
    dx = -p * (dlogp + dent * entropy)[:, None] - dent[:, None] * p * torch.where(there, logs, torch.zeros_like(logs))
    hit = (torch.arange(case["V"], device=x.device) == tok[:, None]) & there
    return out, (dx + hit * dlogp[:, None]).to(s["logits"].dtype)


def _plain_ffn(s, case):
    x, w = s["x"].float(), s["w"].float()
    g, u = x @ w[0].t(), x @ w[1].t()
    if case["act"] == "silu":
        sig = 1.0 / (1.0 + torch.exp(-g))
        act, slope = g * sig, sig * (1.0 + g * (1.0 - sig))
    else:
        k = math.sqrt(2.0 / math.pi)
        t = torch.tanh(k * (g + 0.044715 * g * g * g))
        act = 0.5 * g * (1.0 + t)
        slope = 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * g * g)
    dt = s["x"].dtype
    h = (act * u).to(dt)
    if not case["train"]:
        return h
    dh = s["dh"].float()
    dg, du = dh * u * slope, dh * act
    return h, (dg @ w[0] + du @ w[1]).to(dt), torch.stack((dg.t() @ x, du.t() @ x)).to(dt)


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    d = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}
    return {"norm": _exact_norm, "scan": _exact_scan, "logp": _exact_logp, "ffn": _exact_ffn}[case["op"]](d, case)


def _exact_norm(s, case):
    x, w = s["x"], s["weight"]
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    std = (var + EPS).sqrt()
    hat = (x - mean) / std
    y = torch.addcmul(s["bias"], hat, w)
    if not case["train"]:
        return y
    n = case["n"]
    up = s["dy"] * w
    dx = (n * up - up.sum(1, keepdim=True) - hat * (up * hat).sum(1, keepdim=True)) / (n * std)
    return y, dx, torch.einsum("rn,rn->n", s["dy"], hat), s["dy"].sum(0)


def _exact_scan(s, case):
    """Step by step, forward and back."""
    T, g, v = case["T"], s["gate"], s["value"]
    a = torch.sigmoid(g)
    drop = s["reset"].bool()[:, :, None]
    h, state = torch.empty_like(v), s["h0"]
    for t in range(T):
        state = torch.lerp(v[t], state.masked_fill(drop[t], 0.0), a[t])
        h[t] = state
    if not case["train"]:
        return h, state
    dg, dv = torch.empty_like(g), torch.empty_like(v)
    flow = s["dlast"]
    for t in reversed(range(T)):
        flow = flow + s["dh"][t]
        dv[t] = flow * (1 - a[t])
        held = (h[t - 1] if t else s["h0"]).masked_fill(drop[t], 0.0)
        dg[t] = flow * (held - v[t]) * a[t] * (1 - a[t])
        flow = (flow * a[t]).masked_fill(drop[t], 0.0)
    return h, state, dg, dv, flow


def _exact_logp(s, case):
    x, tok = s["logits"], s["tokens"]
    if s["mask"] is not None:
        x = x.masked_fill(s["mask"] == 0, -math.inf)
    lse = torch.logsumexp(x, 1)
    dead = lse == -math.inf
    logs = (x - lse[:, None]).masked_fill(dead[:, None], -math.inf)
    p = logs.exp()
    entropy = torch.special.entr(p).sum(1)
    absent = (tok < 0) | (tok >= case["V"])
    logp = logs.gather(1, tok.masked_fill(absent, 0)[:, None])[:, 0].masked_fill(absent, 0.0)
    peak = x.amax(1)
    out = dict(logp=logp, entropy=entropy, peak=peak, logz=(lse - peak).masked_fill(dead, -math.inf))
    if case["top"]:
        out["top_logp"], out["top_index"] = logs.topk(case["top"], dim=1).values, None
    if not case["train"]:
        return out
    up = s["dlogp"].masked_fill(absent | dead, 0.0)
    dx = -p * up[:, None] - s["dentropy"][:, None] * p * (logs.masked_fill(p == 0, 0.0) + entropy[:, None])
    dx.scatter_add_(1, tok.masked_fill(absent, 0)[:, None], up[:, None])
    return out, dx.masked_fill(x == -math.inf, 0.0)


def _exact_ffn(s, case):
    x, w, rows, H = s["x"], s["w"].reshape(2 * case["H"], case["D"]), case["rows"], case["H"]
    g, u = (x @ w.t()).reshape(rows, 2, H).unbind(1)
    if case["act"] == "silu":
        act, slope = torch.nn.functional.silu(g), torch.sigmoid(g) + torch.nn.functional.silu(g) * torch.sigmoid(-g)
    else:
        inner = math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
        cdf = torch.sigmoid(2 * inner)
        act, slope = g * cdf, cdf + g * cdf * (1 - cdf) * 2 * math.sqrt(2 / math.pi) * (1 + 0.134145 * g ** 2)
    if not case["train"]:
        return act * u
    both = torch.stack((s["dh"] * u * slope, s["dh"] * act), 1).reshape(rows, 2 * H)
    return act * u, both @ w, (both.t() @ x).reshape(2, H, case["D"])


def work(case):
    """Each input read once, each output written once; operations of the matrix products and, elsewhere, about what
    each value takes."""
    e = 4 if case["dtype"] == "f32" else 2
    train = case["train"]
    if case["op"] == "norm":
        rows, n, pe = case["rows"], case["n"], 4 if case["params"] == "f32" else 2
        return dict(bytes=float(rows * n * e * (4 if train else 2) + n * pe * (4 if train else 2)),
                    flops=float(rows * n * (20 if train else 8)))
    if case["op"] == "scan":
        steps, states = case["T"] * case["B"], case["B"] * case["D"]
        return dict(bytes=float(steps * case["D"] * e * (6 if train else 3) + steps + states * 4 * (4 if train else 2)),
                    flops=float(steps * case["D"] * (20 if train else 6)))
    if case["op"] == "logp":
        rows, V = case["rows"], case["V"]
        return dict(bytes=float(rows * V * (e * (2 if train else 1) + (1 if case["mask"] else 0))
                                + rows * (8 + 12 + 8 * case["top"] + (8 if train else 0))),
                    flops=float(rows * V * (12 if train else 6)))
    rows, D, H = case["rows"], case["D"], case["H"]
    return dict(bytes=float(e * ((2 if train else 1) * (rows * D + 2 * H * D + rows * H))),
                flops=float((12 if train else 4) * rows * D * H))
