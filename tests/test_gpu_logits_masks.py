"""Logits masked with their type's lowest value, and losses whose terms overflow where their factor is 0."""
import numpy as np
import pytest
import torch

import logits_ref as ref
from paper_2606_18967_amd import sdrl
from test_gpu_logits import DT, check_gradient, check_stats, host, policy_inputs, rows, run_policy, y_max

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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [0.6, 1.0, 1.4])
@pytest.mark.parametrize("V", SIZES)
def test_logits_masked_with_the_lowest_value(V, T, dtype):
    x, xh, t, tok = masked(V, dtype, V)
    logp, entropy, norm = sdrl.token_logprobs(x, tok, T)
    check_stats(xh, t, T, logp, entropy, norm)
    g, h = (np.random.default_rng(k).normal(size=8).astype(np.float32) for k in range(2))
    gd, hd = torch.from_numpy(g).cuda(), torch.from_numpy(h).cuda()
    check_gradient(xh, t, T, g, 0 * h, sdrl.token_logprobs_grad(x, tok, norm, gd, T), dtype)
    check_gradient(xh, t, T, g, h, sdrl.token_logprobs_grad(x, tok, norm, gd, T, entropy=entropy, dentropy=hd), dtype)


def check_masked_policy(xh, t, v, kl, ent, T, out, dtype):
    """check_policy's statements and bounds for rows that all have a weight and a token.  (It takes a row of entropy 0 as
    absent, and leaves its terms no rounding; a row with one token left has entropy 0, and counts.)"""
    stats, lp, H, g, h = ref.policy(xh, t, T, v["old"], v["adv"], v["w"], v.get("ref"), v.get("beh"), 0.2, 0.28, kl, ent)
    es = ref.sum_error(xh.shape[1], y_max(xh, T))
    live = np.ones(len(t), bool)
    if "beh" in v:
        f = np.exp(v["old"].astype(np.float64) - v["beh"])
        live = (f >= 0.5) & (f <= 2)
    e_lp = es + ref.E24 * 8 * (np.abs(lp) + 30)
    assert (np.abs(host(out.logp) - lp) <= e_lp).all()
    assert (host(out.logp)[~live] == 0).all() and (host(out.entropy)[~live] == 0).all()
    slope = np.where(live, np.abs(v["w"]) * (np.exp(4) * (np.abs(v["adv"]) + 1) + 1), 0)
    tol = ((e_lp + ref.E24 * 16 + 4 * es * (1 + np.abs(H))) * slope).sum() + ref.E24 * np.abs(stats)
    assert (np.abs(host(out.stats) - stats) <= tol).all(), (host(out.stats), stats, tol)
    if out.dlogits is None:
        return
    d, _ = ref.gradient(xh, t, T, g, h)
    scale = ref.gradient(xh, t, T, slope, h)[1]
    tol = (e_lp[:, None] + es * 4 + ref.E24 * 64) * scale + ref.HALF_STEP[dtype] * np.abs(d) + 1e-38
    off = np.abs(host(out.dlogits) - d)
    assert (off <= tol).all(), np.max(off / tol)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [0.6, 1.0])
@pytest.mark.parametrize("kl,ent", [(0.0, 0.0), (0.05, 0.02)])
@pytest.mark.parametrize("V", SIZES)
def test_policy_loss_of_masked_logits(V, kl, ent, T, dtype):
    x, xh, t, tok = masked(V, dtype, V)
    v = policy_inputs(xh, t, T, V, pad=0.0)
    out = run_policy(x, tok, v, kl, ent, T)
    check_masked_policy(xh, t, v, kl, ent, T, out, dtype)
    less = run_policy(x, tok, v, kl, ent, T, grad=False)
    assert torch.equal(less.stats, out.stats) and torch.equal(less.entropy, out.entropy)


def test_many_rows_of_masked_logits():
    """More rows than are cut into parts, one masked as a whole work-group's first vectors."""
    R, V, T = 300, 70007, 0.8
    x, _ = rows(R, V, "bf16", 1)
    x[::3, :60000] = torch.finfo(torch.bfloat16).min
    t = np.random.default_rng(0).integers(60000, V, R).astype(np.int32)
    tok, xh = torch.from_numpy(t).cuda(), host(x)
    check_stats(xh, t, T, *sdrl.token_logprobs(x, tok, T))
    v = policy_inputs(xh, t, T, 2, pad=0.0)
    check_masked_policy(xh, t, v, 0.05, 0.02, T, run_policy(x, tok, v, 0.05, 0.02, T), "bf16")


@pytest.mark.parametrize("V", [300, 30000, 70001])
@pytest.mark.parametrize("grad", [False, True])
def test_a_ratio_out_of_range_times_an_advantage_of_0_is_0(V, grad):
    """e^(logp - old_logp) past fp32's range at rows whose group's rewards were all alike: their term is 0, as every other
    ratio's, and so is their gradient."""
    x, xh = rows(12, V, "f32", 3)
    t = np.random.default_rng(V).integers(0, V, 12).astype(np.int32)
    v = policy_inputs(xh, t, 1.0, 3, pad=0.0)
    del v["ref"], v["beh"]
    v["old"][::3] -= 300
    v["adv"][::3] = 0
    out = run_policy(x, torch.from_numpy(t).cuda(), v, 0.0, 0.01, 1.0, grad=grad)
    check_masked_policy(xh, t, v, 0.0, 0.01, 1.0, out, "f32")
    v["adv"][3] = np.nan                                          # what is no number stays none
    assert np.isnan(host(run_policy(x, torch.from_numpy(t).cuda(), v, 0.0, 0.01, 1.0, grad=grad).stats)[:2]).all()
