"""Refusals of the calls over logits rows, before anything is launched, and the reference's gradients against
differences.  No GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import logits_ref as ref
from paper_2606_18967_amd import sdrl

BUF = (C.c_char * 8192)()
PTR = (C.addressof(BUF) + 255) & ~255                  # never dereferenced: refused calls launch nothing
INVAL, UNSUPPORTED = sdrl.SD_E_INVAL, sdrl.SD_E_UNSUPPORTED
nan, inf = float("nan"), float("inf")


def test_workspace_bytes():
    f = sdrl.lib().sd_logits_workspace_bytes
    assert f(0, 5) > 0 and f(8, 512) > 0 and f(64, 152064) % 256 == 0
    assert f(-1, 5) == 0 and f(4, 0) == 0 and f((1 << 21) + 1, 5) == 0
    assert f(1, 1 << 30) > 0 and f(1, (1 << 30) + 1) == 0
    with pytest.raises(sdrl.SDError):
        sdrl.logits_workspace_bytes(-1, 5)


@pytest.mark.parametrize("V", [1, 512, 16384, 16385, 50257, 128256, 1 << 30])
def test_a_workspace_serves_fewer_rows_too(V):
    f = sdrl.lib().sd_logits_workspace_bytes
    b = [f(r, V) for r in range(1100)]
    assert b == sorted(b)


def test_vocabularies_past_the_kernels_steps_are_refused():
    V = (1 << 30) + 1                                  # a step past the end of a longer row could pass 2^31
    L, c = sdrl.lib(), sdrl.PolicyCfg(1.0, 0.2, 0.2, 0.0, 0.0, 0.5, 2.0, 0)
    assert L.sd_token_logprobs(0, 1, V, PTR, V, PTR, 1.0, PTR, None, None, PTR, 1 << 40, None) == UNSUPPORTED
    assert L.sd_token_logprobs_grad(0, 1, V, PTR, V, PTR, 1.0, PTR, PTR, None, None, PTR, V, None) == UNSUPPORTED
    assert L.sd_policy_loss(C.byref(c), 0, 1, V, PTR, V, PTR, PTR, None, None, PTR, PTR, PTR, PTR, None, None, 0, PTR, 1 << 40,
                            None) == UNSUPPORTED


COMMON = [dict(dtype=2), dict(rows=-1), dict(V=0), dict(x=None), dict(x=PTR + 2), dict(dtype=1, x=PTR + 1), dict(ld=99), dict(ld=1 << 31),
          dict(tok=None), dict(T=0.0), dict(T=-1.0), dict(T=nan), dict(T=inf), dict(T=1e-39)]


def test_logprobs_are_checked():
    need = sdrl.lib().sd_logits_workspace_bytes(4, 100)

    def call(dtype=0, rows=4, V=100, x=PTR, ld=100, tok=PTR, T=1.0, logp=PTR, ws=PTR, nb=need):
        return sdrl.lib().sd_token_logprobs(dtype, rows, V, x, ld, tok, T, logp, None, None, ws, nb, None)

    for kw in COMMON + [dict(logp=None), dict(ws=None), dict(ws=PTR + 16), dict(nb=need - 1)]:
        assert call(**kw) == INVAL, kw
    assert call(rows=(1 << 21) + 1) == UNSUPPORTED
    assert call(rows=0, x=None, tok=None, logp=None, ws=None, nb=0) == sdrl.SD_OK


def test_logprobs_grad_is_checked():
    def call(dtype=0, rows=4, V=100, x=PTR, ld=100, tok=PTR, T=1.0, norm=PTR, dlogp=PTR, ent=PTR, dent=PTR, out=PTR + 4096, out_ld=100):
        return sdrl.lib().sd_token_logprobs_grad(dtype, rows, V, x, ld, tok, T, norm, dlogp, ent, dent, out, out_ld, None)

    for kw in COMMON + [dict(norm=None), dict(dlogp=None), dict(out=None), dict(ent=None), dict(dent=None), dict(out=PTR + 4097),
                        dict(out_ld=99), dict(out=PTR + 4), dict(out=PTR, out_ld=104), dict(out=PTR + 1596), dict(out=PTR - 1596)]:
        assert call(**kw) == INVAL, kw
    assert call(rows=0, x=None, tok=None, norm=None, dlogp=None, out=None) == sdrl.SD_OK


def test_policy_is_checked():
    need = sdrl.lib().sd_logits_workspace_bytes(4, 100)

    def call(dtype=0, rows=4, V=100, x=PTR, ld=100, tok=PTR, T=1.0, old=PTR, beh=PTR, kl=PTR, adv=PTR, w=PTR, stats=PTR, logp=PTR,
             out=PTR + 4096, out_ld=100, ws=PTR, nb=need, **cfg):
        c = sdrl.PolicyCfg(T, *{**dict(clip_low=0.2, clip_high=0.2, kl_coef=0.1, entropy_coef=0.0, is_low=0.5, is_high=2.0,
                                       reserved=0), **cfg}.values())
        return sdrl.lib().sd_policy_loss(C.byref(c), dtype, rows, V, x, ld, tok, old, beh, kl, adv, w, stats, logp, None, out, out_ld,
                                         ws, nb, None)

    for kw in COMMON + [dict(old=None), dict(kl=None), dict(adv=None), dict(w=None), dict(stats=None), dict(logp=None), dict(ws=None),
                        dict(ws=PTR + 128), dict(nb=need - 1), dict(out=PTR + 4), dict(out_ld=99), dict(clip_low=-0.1),
                        dict(clip_low=1.1), dict(clip_low=nan), dict(clip_high=-0.1), dict(clip_high=inf), dict(clip_high=nan),
                        dict(kl_coef=nan), dict(entropy_coef=inf), dict(is_low=-1.0), dict(is_low=3.0), dict(is_high=nan),
                        dict(reserved=1)]:
        assert call(**kw) == INVAL, kw
    assert sdrl.lib().sd_policy_loss(None, 0, 4, 100, PTR, 100, PTR, PTR, PTR, PTR, PTR, PTR, PTR, PTR, None, None, 0, PTR, need, None) == INVAL
    assert sdrl.lib().sd_last_error()


def test_python_arguments_are_checked(monkeypatch):
    x, t = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        sdrl.token_logprobs(x, t)
    with pytest.raises(ValueError, match="device tensor"):
        sdrl.policy_loss(sdrl.PolicyLoss(), x, t, x[:, 0], x[:, 0], x[:, 0])


def test_reference_gradient_against_differences():
    rng = np.random.default_rng(0)
    x, tok, T = rng.normal(size=(3, 7)) * 2, np.array([2, 0, 6]), 0.7
    g, h = rng.normal(size=3), rng.normal(size=3)
    f = lambda x: (g * ref.logprobs(x, tok, T)[0] + h * ref.logprobs(x, tok, T)[1]).sum()  # noqa: E731
    d, scale = ref.gradient(x, tok, T, g, h)
    for r in range(3):
        for j in range(7):
            e = np.zeros_like(x)
            e[r, j] = 1e-5
            # the third derivatives are below 8 (|g| + |h|) / T^3, and 64 bits leave 1e-11 of a difference
            assert abs((f(x + e) - f(x - e)) / 2e-5 - d[r, j]) < 1e-8
    assert (scale >= np.abs(d) - 1e-15).all()


def test_reference_policy_gradient_against_differences():
    rng = np.random.default_rng(1)
    R, V, T = 12, 9, 1.3
    x, tok = rng.normal(size=(R, V)) * 2, rng.integers(0, V, R)
    lp = ref.logprobs(x, tok, T)[0]
    args = dict(old=lp - rng.normal(size=R) * 0.3, adv=rng.normal(size=R), w=rng.random(R), ref=lp + rng.normal(size=R), kl=0.1, ent=0.05)
    _, _, _, g, h = ref.policy(x, tok, T, **args)
    d, _ = ref.gradient(x, tok, T, g, h)
    for r in range(R):
        for j in range(V):
            e = np.zeros_like(x)
            e[r, j] = 1e-6
            fd = (ref.policy(x + e, tok, T, **args)[0][0] - ref.policy(x - e, tok, T, **args)[0][0]) / 2e-6
            assert abs(fd - d[r, j]) < 1e-7
