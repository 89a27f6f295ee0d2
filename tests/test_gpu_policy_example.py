"""The operators together: the example's recurrent policy acts in the environments and learns from what it did."""
from __future__ import annotations

import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "recurrent_policy.py")
    spec = importlib.util.spec_from_file_location("recurrent_policy", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.fixture(scope="module")
def data(ex):
    import workload as wk
    wl = wk.WORKLOADS[2].scaled(batch=96)
    _, rules, cum = wk.make(wl, 0)
    env = ex.av.Env(dict(wk.config_fields(wl), max_steps=17, auto_reset=1), rules, cum)
    policy = ex.Policy(5 * 5 * env.C, width=64, hidden=136)
    batch = ex.act(env, policy, 40, 5, seed=3)
    env.sync()
    env.close()
    return policy, batch


def test_episodes_end_within_the_trajectory(data):
    _, batch = data
    assert batch["obs"].shape[:2] == (40, 96) and (batch["actions"] < 5).all()
    assert batch["reset"][17].all() and batch["reset"][34].all() and not batch["reset"][0].any()


def test_learning_sees_what_acting_saw(ex, data):
    """Step by step and all at once, the same log probabilities.  Both ways round the same values to bfloat16 at the
    same places; sums in another order move some to the neighbouring value, 2^-8 relatively.  The logits are sums of
    width products of magnitude |x| |head| / sqrt(width) = 0.1 |x|, with |x| below 16 a value: a rounding of every one
    of some six arrays on the way moves a logit by at most 6 x 2^-8 x 0.1 x 16, a log probability by twice that."""
    policy, batch = data
    with torch.no_grad():
        _, logp = ex.loss_of(policy, batch, torch.zeros(40, 96, device="cuda"))
    assert float((logp - batch["logp"]).abs().max()) <= 2 * 6 * 2.0**-8 * 0.1 * 16


def test_steps_along_the_gradient_lower_the_loss(ex, data):
    policy, batch = data
    gain = ex.returns(batch)
    optimiser = torch.optim.SGD(policy.parameters, lr=0.1)
    losses = []
    for _ in range(12):
        loss, _ = ex.loss_of(policy, batch, gain)
        optimiser.zero_grad()
        loss.backward()
        assert all(torch.isfinite(p.grad).all() and p.grad.any() for p in policy.parameters)
        optimiser.step()
        losses.append(float(loss.detach()))
    assert losses[-1] < losses[0]


def test_example_runs(ex):
    assert len(ex.main(updates=2, batch=64, steps=20, window=5)) == 2
