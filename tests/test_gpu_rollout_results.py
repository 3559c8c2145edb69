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


@pytest.mark.parametrize("out", [True, False])
def test_the_command_keeps_log_probabilities(tmp_path, monkeypatch, capsys, out):
    say("rollout --logprobs", out)
    kept = {}
    plain = rollout.Rollout.run

    def spy(self, policy, gamma, tau_prev, cost, eps, lengths, step, keep_trace=True):
        r = plain(self, policy, gamma, tau_prev, cost, eps, lengths, step, keep_trace)
        kept[policy, step] = {k: v.cpu().numpy() if isinstance(v, torch.Tensor) else np.array(v) for k, v in r[1].items() if k in ("tokens", "logp", "gen")}
        kept[policy, step]["lengths"] = np.array(lengths)
        return r

    monkeypatch.setattr(rollout.Rollout, "run", spy)
    calib, to = tmp_path / "calib.json", tmp_path / "run.json"
    calib.write_text(json.dumps(dict(F_eff=1e14, params={}, kv4=False)))
    rollout.main(["--model", "TINY_BF16", "--B", "8", "--prompt", "64", "--lmin", "4", "--lmax", "24", "--median", "12", "--steps", "2",
                  "--policies", "ar,sd", "--calib", str(calib), "--logprobs"] + (["--out", str(to)] if out else []))
    line = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    mean = lambda p, t: np.mean([kept[p, t]["logp"][b, :n].mean(dtype=np.float64) * n for b, n in enumerate(kept[p, t]["lengths"])]) * 8 / kept[p, t]["lengths"].sum()  # noqa: E731
    for p in ("ar", "sd"):
        for t in range(2):
            # sums of at most 192 fp32 values in fp64, however they are ordered
            assert abs(line["mean_logp"][p][t] - mean(p, t)) <= 1e-12 * abs(mean(p, t))
    assert line["logprobs"] is True
    if not out:
        return
    summary = json.loads(to.read_text())
    with np.load(tmp_path / summary["logprobs"], allow_pickle=False) as f:
        for p in ("ar", "sd"):
            for t in range(2):
                for k in ("tokens", "logp", "gen", "lengths"):
                    assert np.array_equal(f[f"{p}_{k}"][t], kept[p, t][k]), (p, t, k)
    assert summary["mean_logp"] == line["mean_logp"]
