"""The policy operators as calls: refusals on GPU tensors, streams, capture in a graph, no state between calls."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pol():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2407_04221_gb300 import policy
    return policy


def inputs(seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, dt=torch.bfloat16: torch.randn(*s, generator=gen, device="cuda").to(dt)  # noqa: E731
    return dict(x=r(500, 256), w=r(256, dt=torch.float32), b=r(256, dt=torch.float32), dy=r(500, 256), g=r(700, 2, 96),
                v=r(700, 2, 96), dh=r(700, 2, 96), reset=(torch.rand(700, 2, generator=gen, device="cuda") < 0.01),
                h0=r(2, 96, dt=torch.float32), logits=r(300, 2000), few=r(3000, 5),
                tok=torch.randint(0, 5, (3000,), generator=gen, device="cuda"), fx=r(300, 128), fw=0.1 * r(2, 264, 128),
                fdh=r(300, 264), one=r(3, 128))


def everything(pol, i, **kw):
    y, m, q = pol.layer_norm(i["x"], i["w"], i["b"], **kw)
    out = [y, *pol.layer_norm_grad(i["dy"], i["x"], i["w"], m, q, **kw)]
    h, last, st = pol.scan(i["g"], i["v"], i["reset"], i["h0"], save=True, **kw)
    out += [h, last, *pol.scan_grad(i["dh"], i["g"], i["v"], i["reset"], st, dlast=i["h0"], **kw)]
    for x in (i["logits"], i["few"]):
        t = i["tok"][:x.shape[0]]
        o = pol.log_probs(x, t, top=4, **kw)
        out += [*o.values(), pol.log_probs_grad(o["logz"], o["logp"], x, t, o, **kw)]
    out += [pol.gated_ffn(i["fx"], i["fw"], **kw), pol.gated_ffn(i["one"], i["fw"], **kw)]
    return out + list(pol.gated_ffn_grad(i["fdh"], i["fx"], i["fw"], **kw))


def test_on_another_stream(pol):
    i = inputs()
    want = everything(pol, i)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        got = everything(pol, i, stream=stream)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(p, q) for p, q in zip(want, got))
    with torch.cuda.stream(side):
        got = everything(pol, i)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_two_streams_at_once(pol):
    """Overlapping calls share nothing."""
    sets = [inputs(k) for k in range(2)]
    want = [everything(pol, i) for i in sets]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(4):
        got = [everything(pol, i, stream=s) for i, s in zip(sets, streams)]
        torch.cuda.synchronize()
        for p, q in zip(want, got):
            assert all(torch.equal(a, b) for a, b in zip(p, q))


def test_captured_in_a_graph(pol):
    i = inputs(3)
    everything(pol, i)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = everything(pol, i)
    other = inputs(4)
    for k in i:
        i[k].copy_(other[k])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(everything(pol, other), got))


def test_inputs_are_left_alone(pol):
    i = inputs(5)
    before = {k: v.clone() for k, v in i.items()}
    everything(pol, i)
    assert all(torch.equal(i[k], before[k]) for k in i)


def test_refusals(pol):
    i = inputs(6)
    cpu = torch.zeros(500, 256)
    x, g, few, fx, fw = i["x"], i["g"], i["few"], i["fx"], i["fw"]
    stats = torch.zeros(500, device="cuda")
    calls = [
        lambda: pol.layer_norm(x.double()), lambda: pol.layer_norm(x.t()), lambda: pol.layer_norm(x, i["w"][:9]),
        lambda: pol.layer_norm(x, i["w"].cpu()), lambda: pol.layer_norm(x, i["w"], i["b"].bfloat16()),
        lambda: pol.layer_norm(x.reshape(50, 10, 256)[:, ::3]), lambda: pol.layer_norm_grad(cpu, x, None, stats, stats),
        lambda: pol.layer_norm_grad(x[:9], x, None, stats, stats), lambda: pol.layer_norm_grad(x, x, None, stats, stats[:4]),
        lambda: pol.scan(g, g[:, :1]), lambda: pol.scan(g, g.float()), lambda: pol.scan(g[0], g[0]),
        lambda: pol.scan(g, g, i["reset"].int()), lambda: pol.scan(g, g, i["reset"][:9]),
        lambda: pol.scan(g, g, None, i["h0"].bfloat16()), lambda: pol.scan(g, g, None, i["h0"].t()),
        lambda: pol.scan(g.transpose(1, 2), g.transpose(1, 2)), lambda: pol.scan_grad(g, g, g, None, stats),
        lambda: pol.log_probs(few, i["tok"][:9]), lambda: pol.log_probs(few, i["tok"].float()),
        lambda: pol.log_probs(few, i["tok"], top=6), lambda: pol.log_probs(few, i["tok"], top=-1),
        lambda: pol.log_probs(i["logits"], i["tok"][:300], top=33), lambda: pol.log_probs(few, i["tok"], mask=few),
        lambda: pol.log_probs(few, i["tok"], mask=torch.ones(4, dtype=torch.uint8, device="cuda")),
        lambda: pol.log_probs_grad(stats, None, few, i["tok"], pol.log_probs(few, i["tok"])),
        lambda: pol.gated_ffn(fx, fw, act="relu"), lambda: pol.gated_ffn(fx.float(), fw.float()),
        lambda: pol.gated_ffn(fx, fw.half()), lambda: pol.gated_ffn(fx, fw[:, :, :64]), lambda: pol.gated_ffn(fx, fw[0]),
        lambda: pol.gated_ffn(fx, fw.transpose(1, 2)), lambda: pol.gated_ffn_grad(i["fdh"][:9], fx, fw),
    ]
    for k, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(f"call {k} was not refused")
    import paper_2407_04221_gb300 as av
    for call in (lambda: pol.gated_ffn(fx[:, 1:65], fw[:, :, :64].contiguous()),  # not 16-byte aligned
                 lambda: pol.gated_ffn(fx[:, :60], fw[:, :, :60].contiguous()),   # not a multiple of 8
                 lambda: pol.gated_ffn(fx[:1].expand(30, 128), fw),               # rows not apart
                 lambda: pol.layer_norm(x, eps=-1.0)):
        with pytest.raises(av.AvError) as err:
            call()
        assert err.value.status == av.AV_EINVAL
