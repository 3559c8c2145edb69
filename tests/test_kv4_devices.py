"""The 4-bit cache's engine calls refuse an engine of another device than the current one: they allocate and launch there.
No GPU: an engine object without its handle."""
import types

import pytest
import torch

from paper_2606_18967_amd import sdrl


@pytest.mark.parametrize("call", ["set_rope", "bind_kv4"])
def test_an_engine_of_another_device_is_refused(monkeypatch, call):
    eng = object.__new__(sdrl.Engine)
    eng.device, eng.h = torch.device("cuda", 1), None
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(sdrl, "lib", lambda: pytest.fail("reached the library"))
    arg = sdrl.RopeConfig(1e4, 64) if call == "set_rope" else types.SimpleNamespace(device=eng.device, _ref=None)
    with pytest.raises(ValueError, match="current device is cuda:0"):
        getattr(eng, call)(arg)
