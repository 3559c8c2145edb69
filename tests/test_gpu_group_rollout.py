"""Groups of rollouts through the engine: steps on shared prompts against the same engine without sharing, the
rollout driver's groups and log-probabilities, and a run from rollout to policy gradient."""
import numpy as np
import pytest
import torch

import logits_ref as ref
from gpu_common import say
from paper_2606_18967_amd import rollout, sdrl, synth

pytestmark = pytest.mark.gpu
GQA = dict(name="grouped-bf16", n_layers=2, hidden=512, n_q=4, n_kv=2, head_dim=128, ffn=1024, vocab=2048, dtype="bf16",
           rope_theta=500000.0, rms_eps=1e-5)
SMALL = dict(GQA, name="grouped-bf16-d64", n_q=8, n_kv=2, head_dim=64, vocab=512)
TOL = 4e-2                      # two engines, each within the 2e-2 that bf16 logits are held to


def grouped(cfg, B, group, prompt, room, gamma, seed=3):
    eng = sdrl.Engine(cfg, B, prompt + room, gamma)
    eng.bind_weights([w.cuda() for w in synth.make_weights(cfg, seed, "cpu")])
    table, gid, n_pages = rollout.grouped_tables(B, group, 0, prompt, prompt + room, 64)
    k, v, kv_len = eng.alloc_kv_paged(n_pages, 64)
    table = torch.from_numpy(table).cuda()
    eng.bind_kv_paged(k, v, table, kv_len)
    k.normal_(), v.normal_()
    if prompt % 64:
        own = table[:, prompt // 64].long()
        for t in (k, v):
            t[own, :, :, :prompt % 64] = t[own[torch.arange(B).cuda() // group * group], :, :, :prompt % 64]
    kv_len.fill_(prompt)
    groups = sdrl.PrefixGroups(torch.from_numpy(gid).cuda(), torch.full((B // group,), prompt, dtype=torch.int32, device="cuda"))
    eng.refresh_drafter()
    return eng, (k, v, kv_len, table), groups


def near(a, b):
    a, b = a.double().flatten(0, -2), b.double().flatten(0, -2)
    rel = (a - b).norm(dim=1) / b.norm(dim=1)
    assert float(rel.max()) < TOL, float(rel.max())


@pytest.mark.parametrize("cfg,prompt", [(GQA, 203), (GQA, 64), (SMALL, 130), (SMALL, 20)], ids=lambda x: str(x if isinstance(x, int) else x["name"]))
def test_steps_with_shared_prompts(cfg, prompt):
    B, group, gamma, T = 8, 4, 4, 1.0
    say("grouped", cfg["name"], prompt)
    eng, (k, v, kv_len, table), groups = grouped(cfg, B, group, prompt, 64, gamma)
    slots = torch.arange(B, dtype=torch.int32, device="cuda")
    last = synth.make_tokens(B, 1, cfg["vocab"], 1)[:, 0].cuda().contiguous()
    draft = synth.make_tokens(B, gamma, cfg["vocab"], 2).cuda().contiguous()
    kv_len += torch.arange(B, dtype=torch.int32, device="cuda") * 3          # responses of different lengths
    keep_k, keep_v, lens = k.clone(), v.clone(), kv_len.clone()
    got = {}
    for on in (False, True):
        k.copy_(keep_k), v.copy_(keep_v), kv_len.copy_(lens)
        eng.bind_prefix(groups if on else None)
        p = torch.zeros((B, gamma + 1, cfg["vocab"]), device="cuda")
        eng.verify(slots, last, draft, gamma, p)
        cached = k.clone(), v.clone()
        a, out = torch.zeros((B, cfg["vocab"]), device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
        eng.ar_step(slots, last, T, 5, 6, out, a)
        kv_len.copy_(lens)
        bufs = sdrl.SDBuffers(eng, B, 1)
        eng.draft(slots, last, 1, T, 5, 6, bufs.draft_tok, bufs.q_logits, bufs.q_stats)
        eng.sync()
        got[on] = p, a, bufs.q_logits, cached
    for x, y in zip(got[True][:3], got[False][:3]):
        near(x, y)
        assert not torch.equal(x, y) or prompt < 64                           # another kernel ran
    # the first layer's new keys and values come of the same rows: rounded once, from fp32 sums of one rounding each
    for x, y in zip(got[True][3], got[False][3]):
        assert ((x[:, 0].float() - y[:, 0].float()).abs() <= 2.0 ** -7 * y[:, 0].float().abs() + 1e-6).all()
    eng.close()


def test_a_shrinking_reordered_batch():
    """Slots that leave and change places, as a rollout's do, step by step against the engine without groups."""
    B, group, gamma, cfg = 8, 4, 3, GQA
    say("grouped, shrinking batch")
    eng, (k, v, kv_len, table), groups = grouped(cfg, B, group, 190, 64, gamma)
    for ids in ([0, 1, 2, 3, 4, 5, 6, 7], [1, 3, 4, 5, 7], [7, 2, 3, 0], [6], [5, 0]):
        slots = torch.tensor(ids, dtype=torch.int32, device="cuda")
        last = synth.make_tokens(len(ids), 1, cfg["vocab"], len(ids))[:, 0].cuda().contiguous()
        draft = synth.make_tokens(len(ids), gamma, cfg["vocab"], 2).cuda().contiguous()
        p = [torch.zeros((len(ids), gamma + 1, cfg["vocab"]), device="cuda") for _ in range(2)]
        for on in (0, 1):
            eng.bind_prefix(groups if on else None)
            eng.verify(slots, last, draft, gamma, p[on])
        eng.sync()
        near(p[1], p[0])
        eng.rollback(slots, torch.full((len(ids),), 2, dtype=torch.int32, device="cuda"))
    eng.close()


def test_bind_prefix_refusals():
    g = sdrl.PrefixGroups(torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"))
    eng = sdrl.Engine(synth.TINY, 4, 64, 2)
    kp, vp, ln = eng.alloc_kv_paged(8, 32)
    table = torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    eng.bind_kv_paged(kp, vp, table, ln)
    with pytest.raises(sdrl.SDError) as ei:
        eng.bind_prefix(g)
    assert ei.value.status == sdrl.SD_E_UNSUPPORTED
    eng.close()
    eng = sdrl.Engine(GQA, 4, 64, 2)
    for bind in (lambda: None, lambda: eng.bind_kv(*eng.alloc_kv()), lambda: eng.bind_kv4(eng.alloc_kv4(8, 32, table))):
        bind()
        with pytest.raises(sdrl.SDError) as ei:
            eng.bind_prefix(g)
        assert ei.value.status == sdrl.SD_E_STATE
    with pytest.raises(ValueError):
        eng.bind_prefix(sdrl.PrefixGroups(torch.zeros(5, dtype=torch.int32, device="cuda"), g.length))
    eng.bind_prefix(None)
    eng.close()


def test_flags_of_grouped_steps():
    eng, (k, v, kv_len, table), groups = grouped(GQA, 4, 2, 128, 64, 2)
    eng.bind_prefix(groups)
    last = torch.zeros(4, dtype=torch.int32, device="cuda")
    out, lg = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros((4, GQA["vocab"]), device="cuda")
    slots = torch.tensor([0, 1, 2, 9], dtype=torch.int32, device="cuda")
    eng.ar_step(slots, last, 1.0, 1, 1, out, lg)
    with pytest.raises(sdrl.SDError, match="slot"):
        eng.sync()
    table[0, 1] = 1 << 20
    eng.ar_step(slots[:3].contiguous(), last[:3].contiguous(), 1.0, 1, 1, out[:3], lg[:3])
    with pytest.raises(sdrl.SDError, match="block-table"):
        eng.sync()
    eng.close()


@pytest.fixture(scope="module")
def ro():
    r = rollout.Rollout(SMALL, B=8, prompt=150, lmax=40, seed=5, group=4, prefill=True, logprobs=True)
    yield r
    r.close()


@pytest.mark.parametrize("policy,gamma", [("ar", 5), ("sd", 5), ("toggle", 7)])
def test_rollout_of_groups_keeps_log_probabilities(ro, policy, gamma, monkeypatch):
    say("grouped rollout", policy, gamma)
    calls = []
    plain = sdrl.token_logprobs

    def spy(logits, tokens, T, workspace=None):
        r = plain(logits, tokens, T, workspace=workspace)
        lp, _, _ = ref.logprobs(logits.double().flatten(0, -2).cpu().numpy(), tokens.flatten().cpu().numpy(), T)
        tol = ref.sum_error(logits.shape[-1], 40) + ref.E24 * 8 * (np.abs(lp) + 30)
        assert (np.abs(r[0].double().flatten().cpu().numpy() - lp) <= tol).all()
        calls.append((tokens.clone(), r[0].clone()))
        return r

    monkeypatch.setattr(sdrl, "token_logprobs", spy)
    L = np.array([3, 19, 1, 37, 5, 12, 40, 8])
    res, st = ro.run(policy, gamma, 5.0, sdrl.cost_init(ro.cfg), 0.05, L, step=1)
    assert (st["gen"] >= L).all() and (ro.kv_len.cpu().numpy() - ro.prompt == st["gen"]).all()
    live = np.arange(8)
    toks, lps = [[] for _ in range(8)], [[] for _ in range(8)]
    for t, lp in calls:
        for row, b in enumerate(live):
            n = int((t[row] >= 0).sum())
            toks[b] += t[row, :n].tolist()
            lps[b] += lp[row, :n].tolist()
        live = np.array([b for b in live if len(toks[b]) < L[b]])
    for b in range(8):
        m = int(st["gen"][b])
        assert len(toks[b]) == m and st["tokens"][b, :m].tolist() == toks[b] and st["logp"][b, :m].tolist() == lps[b]


def test_graph_rollout_of_groups_equals_eager():
    say("grouped rollout with graphs")
    L = np.array([30, 2, 11, 7, 25, 19])
    got = []
    for graphs in (False, True):
        r = rollout.Rollout(SMALL, B=6, prompt=140, lmax=30, seed=5, group=3, graphs=graphs, padded=True, logprobs=True)
        res, st = r.run("sd", 5, 5.0, sdrl.cost_init(r.cfg), 0.05, L, step=3)
        got.append((st["gen"].tolist(), st["tokens"].cpu(), st["logp"].cpu()))
        r.close()
    for b, m in enumerate(got[0][0]):
        assert got[1][0][b] == m and torch.equal(got[0][1][b, :m], got[1][1][b, :m]) and torch.equal(got[0][2][b, :m], got[1][2][b, :m])


def test_groups_and_the_4_bit_cache():
    with pytest.raises(ValueError, match="4-bit"):
        rollout.Rollout(SMALL, B=4, prompt=64, lmax=8, group=2, kv4=True)


def test_from_rollout_to_policy_gradient(ro):
    """Rollout of groups, the learner's logits of its responses, advantages within a group, the loss and its gradient."""
    say("rollout to policy gradient")
    gamma, T, cfg = 5, ro.T, ro.cfg
    L = np.array([6, 9, 6, 30, 7, 12, 40, 8])
    res, st = ro.run("sd", gamma, 5.0, sdrl.cost_init(cfg), 0.05, L, step=2)
    # the logits of the first gamma + 1 response tokens, teacher-forced through the grouped engine
    n = gamma + 1
    ro.kv_len.fill_(ro.prompt)
    last = synth.make_tokens(8, 1, cfg["vocab"], ro.seed + 7 + 2)[:, 0].cuda().contiguous()
    logits = torch.zeros((8, n, cfg["vocab"]), device="cuda")
    tokens = st["tokens"][:, :n].contiguous()
    slots = torch.arange(8, dtype=torch.int32, device="cuda")
    ro.eng.verify(slots, last, tokens[:, :gamma].contiguous(), gamma, logits)
    ro.eng.sync()
    behavior = st["logp"][:, :n].contiguous()
    old, _, _ = sdrl.token_logprobs(logits, tokens, T)
    # the rollout's own logits are this engine's at other batch shapes: both within 2e-2 of the exact ones
    assert float((old - behavior).abs().max()) <= 2 * TOL * float(logits.abs().max())
    reward = torch.tensor([1.0, 0, 0, 1, 0, 0, 1, 0], device="cuda").view(2, 4)
    adv = ((reward - reward.mean(1, keepdim=True)) / (reward.std(1, keepdim=True) + 1e-6)).view(8, 1).expand(8, n).contiguous()
    weight = (torch.arange(n, device="cuda")[None] < torch.from_numpy(L).cuda()[:, None]).float()
    weight = weight / weight.sum()
    refp = old - 0.1
    out = sdrl.policy_loss(sdrl.PolicyLoss(0.2, 0.28, 0.1, 0.01, temperature=T), logits, tokens, old, adv, weight, ref_logp=refp,
                           behavior_logp=behavior)
    h = lambda t: t.double().flatten().cpu().numpy()  # noqa: E731
    x, t = logits.double().flatten(0, 1).cpu().numpy(), tokens.flatten().cpu().numpy()
    stats, lp, H, g, dh = ref.policy(x, t, T, h(old), h(adv), h(weight), h(refp), h(behavior), 0.2, 0.28, 0.1, 0.01)
    e = ref.sum_error(cfg["vocab"], 40) * 8 + ref.E24 * 64 * 30
    assert np.abs(h(out.stats) - stats).max() <= e * 8 and stats[4] == 0      # the ratio is 1: nothing is clipped
    d, scale = ref.gradient(x, t, T, np.abs(h(weight)) * 4, dh)
    want = ref.gradient(x, t, T, g, dh)[0]
    assert (np.abs(h(out.dlogits).reshape(want.shape) - want) <= e * scale * 4 + 1e-12).all()
