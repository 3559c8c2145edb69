"""Logits masked with their type's lowest value, and losses whose terms overflow where their factor is 0."""
import numpy as np
import pytest
import torch

import logits_ref as ref
from paper_2606_18967_amd import sdrl
from test_gpu_logits import DT, check_gradient, check_policy, check_stats, host, policy_inputs, rows, run_policy

pytestmark = pytest.mark.gpu
# whole vectors of few rows and many, a lone tail, parts of a row
SIZES = [1, 5, 9, 129, 4099, 40000, 70007, 131075]


def masked(V, dtype, seed):
    """Rows of which most, the first three quarters, the second half, all but the last, all and every second of the logits
    are the type's lowest value, a row with a large finite mask, and one without a mask; tokens that are not masked."""
    x, _ = rows(8, V, dtype, seed)
    low = torch.finfo(DT[dtype]).min
    t = np.array([V // 3, V - 1, 0, V - 1, V // 2, 0, V - 1, V // 5], np.int32)
    x[0] = low
    x[0, V // 3] = 1.5
    x[1, :3 * V // 4] = low
    x[2, (V + 1) // 2:] = low
    x[3, :V - 1] = low
    x[4] = low
    x[5, 1::2] = low
    x[6, :3 * V // 4] = -2.5e38
    return x, host(x), t, torch.from_numpy(t).cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [0.6, 1.0])
@pytest.mark.parametrize("V", SIZES)
def test_a_loss_without_an_entropy_term_does_not_depend_on_the_entropy(V, T, dtype):
    x, xh, t, tok = masked(V, dtype, V)
    v = policy_inputs(xh, t, T, V, pad=0.0)
    for grad in (False, True):
        stats = host(run_policy(x, tok, v, 0.0, 0.0, T, grad=grad).stats)
        assert np.isfinite(stats[0]) and stats[0] == stats[1]      # the loss is its clipped term alone
