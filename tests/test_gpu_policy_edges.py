"""The policy operators at their edges: NaN among the alternatives of long rows."""
from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")

from tests import test_gpu_policy_logp as logp  # noqa: E402
from tests.policy_ref import BF16, F32, top_of  # noqa: E402

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
