"""What a rollout leaves of its responses: tokens and log-probabilities of its own, and what the command keeps."""
import json

import numpy as np
import pytest
import torch

from gpu_common import say
from paper_2606_18967_amd import rollout, sdrl, synth

pytestmark = pytest.mark.gpu
CFG = dict(synth.TINY, dtype="bf16", name="tiny-bf16")


@pytest.mark.parametrize("group", [1, 4])
def test_results_outlive_the_next_run(group):
    say("two rollouts", group)
    r = rollout.Rollout(CFG, B=8, prompt=70, lmax=40, seed=5, group=group, logprobs=True)
    cost = sdrl.cost_init(CFG)
    first = r.run("sd", 5, 5.0, cost, 0.05, np.array([40, 40, 1, 40, 5, 40, 40, 40]), step=1)[1]
    tokens, logp = first["tokens"].clone(), first["logp"].clone()
    L = np.array([3, 19, 1, 37, 5, 12, 40, 8])
    second = r.run("ar", 5, 5.0, cost, 0.05, L, step=2)[1]
    assert torch.equal(first["tokens"], tokens) and torch.equal(first["logp"], logp)
    assert not torch.equal(second["tokens"], tokens)
    for st in (first, second):
        assert st["tokens"].shape == st["logp"].shape and st["tokens"].shape[0] == 8 and st["tokens"].shape[1] >= 40
        past = torch.arange(st["tokens"].shape[1], device="cuda")[None] >= torch.from_numpy(st["gen"]).cuda()[:, None]
        assert (st["tokens"][past] == -1).all() and (st["logp"][past] == 0).all()
        assert (st["tokens"][~past] >= 0).all() and (st["logp"][~past] < 0).all()
    r.close()
