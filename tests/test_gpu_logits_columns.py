"""Logits and their gradient as columns of one buffer."""
import numpy as np
import pytest
import torch

from paper_2606_18967_amd import sdrl
from test_gpu_logits import DT, check_gradient, check_policy, host, policy_inputs, rows, run_policy, tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,V", [(7, 129), (5, 4099), (6, 70007), (300, 515)])
@pytest.mark.parametrize("first", [True, False])
def test_gradient_beside_the_logits(R, V, first, dtype):
    x, xh = rows(R, V, dtype, V)
    buf = torch.full((R, 2 * V + 3), 7.0, dtype=DT[dtype], device="cuda")
    a, b = buf[:, :V], buf[:, V + 1:2 * V + 1]
    x, out = (a.copy_(x), b) if first else (b.copy_(x), a)
    t, tok = tokens(R, V, V)
    _, _, norm = sdrl.token_logprobs(x, tok)
    g = np.ones(R, np.float32)
    sdrl.token_logprobs_grad(x, tok, norm, torch.ones(R, device="cuda"), out=out)
    check_gradient(xh, t, 1.0, g, 0 * g, out, dtype)
    v = policy_inputs(xh, t, 1.0, R)
    check_policy(xh, t, v, 0.05, 0.02, 1.0, run_policy(x, tok, v, 0.05, 0.02, 1.0, dlogits=out), dtype)
    assert np.array_equal(host(x), xh) and (buf[:, V] == 7).all() and (buf[:, 2 * V + 1:] == 7).all()
