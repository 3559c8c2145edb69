"""Calibrations say which kind of KV cache they were made on, and a rollout takes only its own kind.  Host logic, with
stand-ins for the GPU's times."""
import json

import pytest

from paper_2606_18967_amd import calibrate, rollout, sdrl, synth

TRUTH = dict(BW_eff=5.2e12, rho_kappa=0.8, c_T=2e-6, eta_D=1.3, c_D=1.5e-6, c_V=3e-6)
CALIB = dict(F_eff=7.0e14, params=dict(BW_eff=5.0e12, rho_kappa=0.9, eta_D=0.95, c_T=1e-6, c_D=2e-6, c_V=3e-6))


class FakeSweep:
    made = []

    def __init__(self, cfg, Bmax, Smax, gmax, seed=2, fmt="w4", kv4=False):
        FakeSweep.made.append(kv4)
        self.base = sdrl.cost_init(cfg, kv_bytes=sdrl.kv4_bytes_per_element(cfg["head_dim"]) if kv4 else 2.0)
        self.base.F_eff = 1.6e15

    def set_drafter(self, fmt):
        pass

    def measure(self, B, S, gammas, reps=8):
        tp, tq, _ = calibrate.model_times(self.base, TRUTH, B, S, 1)
        return {"p": tp, "q": tq, **{("v", g): calibrate.model_times(self.base, TRUTH, B, S, g)[2] for g in gammas}}

    def measured_tau(self, B, S, gamma, steps=10):
        return 2.5

    def close(self):
        pass


@pytest.fixture
def fake(monkeypatch):
    FakeSweep.made = []
    monkeypatch.setattr(calibrate, "Sweep", FakeSweep)
    monkeypatch.setattr(calibrate, "f_eff", lambda *a, **k: 1.6e15)


@pytest.mark.parametrize("kv4", [False, True])
def test_a_calibration_names_its_cache_and_drafter(fake, kv4):
    res = calibrate.run(synth.L32_8B, [1, 4, 16, 64], [512, 2048, 8192], [3, 7], [2.0, 4.0], log=lambda *a: None, fmt="w8", kv4=kv4)
    assert FakeSweep.made == [kv4] and res["kv4"] is kv4 and res["drafter"] == "w8"
    m = rollout.calibrated_cost(synth.L32_8B, json.loads(json.dumps(res, default=str)), kv4)
    assert m.BW_eff == pytest.approx(res["params"]["BW_eff"])
    with pytest.raises(ValueError, match="calibration"):
        rollout.calibrated_cost(synth.L32_8B, res, not kv4)


def test_a_calibration_that_does_not_say_is_of_the_models_cache():
    assert rollout.calibrated_cost(synth.L4_8B, CALIB).F_eff == 7.0e14
    with pytest.raises(ValueError, match="4-bit"):
        rollout.calibrated_cost(synth.L4_8B, CALIB, True)


@pytest.mark.parametrize("of", [None, False, True])
def test_the_rollout_command_refuses_the_other_kind(tmp_path, of):
    """Before it builds an engine."""
    path = tmp_path / "calib.json"
    path.write_text(json.dumps(CALIB if of is None else dict(CALIB, kv4=of)))
    argv = ["--model", "TINY_BF16", "--calib", str(path)] + ([] if of else ["--kv4"])
    with pytest.raises(ValueError, match="calibration"):
        rollout.main(argv)


@pytest.mark.parametrize("kv4", [False, True])
def test_the_drafter_comparison_runs_on_the_cache_that_is_asked_for(fake, capsys, kv4):
    calibrate.main(["--drafter-tradeoff", "--B", "1,4", "--S", "512", "--gamma", "3"] + (["--kv4"] if kv4 else []))
    rows = json.loads(capsys.readouterr().out)
    assert FakeSweep.made == [kv4] and len(rows) == 6 and all(r["kv4"] is kv4 for r in rows)
    ideal = sdrl.cost_init(synth.L4_8B, kv_bytes=sdrl.kv4_bytes_per_element(128) if kv4 else 2.0, BW_eff=1.0, F_eff=1e30)
    tp, tq, _ = sdrl.cost_times(ideal, 4, 512, 3)
    assert rows[1]["tq_over_tp_ideal"] == pytest.approx(tq / tp)
