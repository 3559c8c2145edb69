"""The engine on a 4-bit KV cache: ragged prefill, drafts, verify, AR steps and rollback against a 64-bit decoder
over the same format (kv4_ref.Decoder), page order, graphs, poisoned rows, scaled rotary tables, and what
sd_bind_kv4 refuses."""
import ctypes as C

import numpy as np
import pytest
import torch

import kv4_ref as ref
import oracle
from oracle.parity import check_accept, check_draws, row_tol_ok
from paper_2606_18967_amd import sdrl, synth

from gpu_common import check_invariants, host_bits, host_bufs, i32, make_engine, say, step_arrays

pytestmark = pytest.mark.gpu

GQA = dict(name="kv4-128", n_layers=2, hidden=512, n_q=4, n_kv=2, head_dim=128, ffn=1024, vocab=2048, dtype="bf16",
           rope_theta=500000.0, rms_eps=1e-5)
MHA = dict(name="kv4-64", n_layers=2, hidden=256, n_q=4, n_kv=4, head_dim=64, ffn=512, vocab=512, dtype="bf16",
           rope_theta=10000.0, rms_eps=1e-5)
LONG = dict(scaling="llama3", factor=8.0, low=1.0, high=4.0, orig_ctx=64)


def setup(cfg, W, slots, max_ctx, gamma, page=32, seed=0, fmt="w4", rope=None, order=True):
    eng = sdrl.Engine(cfg, slots, max_ctx, gamma)
    eng.bind_weights(W)
    if rope is not None:
        eng.set_rope(rope)
    per = -(-max_ctx // page)
    g = torch.Generator().manual_seed(seed)
    table = torch.randperm(slots * per + 2, generator=g)[:slots * per] if order else torch.arange(slots * per)
    cache = eng.alloc_kv4(slots * per + 2, page, table.to(torch.int32).reshape(slots, per).cuda())
    eng.bind_kv4(cache)
    eng.refresh_drafter(fmt=fmt)
    return eng, cache


def decoders(cfg, W, table, fmt="w4"):
    host = host_bits(W)
    w = [oracle.tensor_f32(t, oracle.BF16).astype(np.float64) for t in host]
    target = [tuple(w[3 + 6 * l + i] for i in (1, 2, 4, 5)) for l in range(cfg["n_layers"])]

    def deq(x):
        codes, sc, zeros = oracle.quantize(x.astype(np.float32), fmt)
        s = oracle.f16_bits_to_f32(sc).astype(np.float64)
        c = codes.astype(np.float64) - (0 if zeros is None else np.repeat(zeros, 128, 1).astype(np.float64))
        return c * np.repeat(s, 128, 1)

    draft = [tuple(deq(x) for x in p) for p in target]
    return ref.Decoder(cfg, w, target, table), ref.Decoder(cfg, w, draft, table, half=True)


def table_of(cfg, n, rope=None):
    f, _ = ref.frequencies(cfg["rope_theta"], cfg["head_dim"], **(rope or {}))
    ang = np.arange(n)[:, None] * f
    return np.stack((np.cos(ang), np.sin(ang)), -1).astype(np.float32)


def values(cache, cfg, slot, n):
    """K and V [L][n_kv][n][D] of a slot's first n positions, as their codes stand for."""
    hc = ref.HostCache(cache.pages.cpu().numpy(), cache.block_table.cpu().numpy(), cache.head_dim)
    out = []
    for is_v in (False, True):
        rows = [[hc.rows(slot, l, h, n, is_v) for h in range(cfg["n_kv"])] for l in range(cfg["n_layers"])]
        out.append((np.array([[z[:, None] + s[:, None] * c for c, s, z in r] for r in rows]),
                    np.array([[s for _, s, _ in r] for r in rows])))
    return out


@pytest.mark.parametrize("cfg,fmt,rope", [(GQA, "w4", None), (MHA, "w8", None), (GQA, "w4a", LONG), (MHA, "w4", LONG)],
                         ids=["gqa", "mha", "gqa-scaled", "mha-scaled"])
def test_steps_against_64_bits(cfg, fmt, rope):
    """Prefill rows are the reference's but for single codes (a value within the GEMM's rounding of a border); on the
    device's own cached rows every draft, verify and AR logit row is within the framework's bf16 bound of 2e-2."""
    say("kv4 engine", cfg["name"], fmt, rope)
    B, gamma, T, seed = 3, 4, 1.0, 5
    lens, cap = [37, 64, 5], 64 + 4 * (gamma + 1) + 4
    W = synth.make_weights(cfg, seed, "cpu", std=0.05)
    rc = None if rope is None else sdrl.RopeConfig(cfg["rope_theta"], cfg["head_dim"], rope["scaling"], rope["factor"],
                                                   rope["low"], rope["high"], rope["orig_ctx"])
    eng, cache = setup(cfg, [w.cuda() for w in W], B, cap, gamma, fmt=fmt, rope=rc)
    rr = None if rope is None else dict(scaling=rope["scaling"], factor=rope["factor"], low=rope["low"], high=rope["high"],
                                        orig=rope["orig_ctx"])
    target, draft = decoders(cfg, W, table_of(cfg, cap, rr), fmt)
    tok = synth.make_tokens(B, 65, cfg["vocab"], seed)
    slots = i32([2, 0, 1])
    eng.prefill_ragged(slots, tok[:, :64].cuda().contiguous(), i32(lens))
    eng.sync()
    L, H, D = cfg["n_layers"], cfg["n_kv"], cfg["head_dim"]
    K, V = np.zeros((3, L, H, cap, D)), np.zeros((3, L, H, cap, D))
    for b, slot in enumerate((2, 0, 1)):
        n = lens[b]
        target.forward(tok[b, :n].numpy(), 0, K[slot], V[slot])
        for (got, s), want in zip(values(cache, cfg, slot, n), (K, V)):
            d = np.abs(got - want[slot][:, :, :n])
            # layer 0 sees exact embeddings: a step at most, from a border crossed or s, z rounded the other way
            assert (d[0] <= 1.3 * s[0][..., None] + 1e-6).all()
            assert (d[0] > 0.5 * s[0][..., None]).mean() < 0.02, float((d[0] > 0.5 * s[0][..., None]).mean())
    kv = [lens[b] for b in range(B)]
    last = i32([int(tok[b, lens[b]]) for b in range(B)])
    bufs = sdrl.SDBuffers(eng, B, gamma)
    worst = 0.0
    order = (2, 0, 1)

    def caches(slot, n):
        """The device's first n rows of a slot with their steps, padded to cap."""
        out = []
        for val, st in values(cache, cfg, slot, n):
            x, y = np.zeros((L, H, cap, D)), np.zeros((L, H, cap))
            x[:, :, :n], y[:, :, :n] = val, st
            out += [x, y]
        return out[0], out[2], (out[1], out[3])

    def close(got, want, at):
        ok, rel = row_tol_ok(got, want, 2e-2)
        assert ok, (at, rel)
        return rel

    for step in range(2):
        eng.draft(slots, last, gamma, T, seed, step, bufs.draft_tok, bufs.q_logits, bufs.q_stats)
        eng.sync()
        first, drafts = last.cpu().numpy(), bufs.draft_tok.cpu().numpy()
        for b, slot in enumerate(order):
            toks = np.concatenate((first[b:b + 1], drafts[b]))
            k, v, st = caches(slot, kv[b] + gamma)
            for j in range(gamma):
                worst = max(worst, close(bufs.q_logits[b, j].cpu().numpy(),
                                         draft.forward(toks[j:j + 1], kv[b] + j, k, v, st)[0], ("draft", step, b, j)))
        eng.verify(slots, last, bufs.draft_tok, gamma, bufs.p_logits)
        eng.sync()
        for b, slot in enumerate(order):
            toks = np.concatenate((first[b:b + 1], drafts[b]))
            k, v, st = caches(slot, kv[b] + gamma + 1)
            p = target.forward(toks, kv[b], k, v, st)
            for j in range(gamma + 1):
                worst = max(worst, close(bufs.p_logits[b, j].cpu().numpy(), p[j], ("verify", step, b, j)))
        eng.accept(slots, bufs.draft_tok, bufs.q_logits, bufs.q_stats, bufs.p_logits, gamma, T, seed, step, bufs.out_tok,
                   bufs.n_emit, bufs.next_tok)
        eng.rollback(slots, bufs.n_emit)
        eng.sync()
        last = bufs.next_tok.clone()
        h = host_bufs(bufs)
        for b, slot in enumerate(order):
            dv = step_arrays(h, b)
            check_invariants(dv, gamma)
            check_draws(dv["q"], dv["draft"], T, (seed, step, slot, kv[b]), dv["q_stats"])
            check_accept(dv, T, (seed, step, slot, kv[b]))
            kv[b] += dv["n_emit"]
    assert cache.kv_len.cpu().tolist() == [kv[1], kv[2], kv[0]]
    out, lg = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros((B, cfg["vocab"]), device="cuda")
    eng.ar_step(slots, last, T, seed, 9, out, lg)
    eng.sync()
    for b, slot in enumerate(order):
        k, v, st = caches(slot, kv[b] + 1)
        worst = max(worst, close(lg[b].cpu().numpy(), target.forward(last[b:b + 1].cpu().numpy(), kv[b], k, v, st)[0], ("ar", b)))
    say("worst relative logit error", worst)
    eng.close()


def run_steps(eng, cache, cfg, n_steps, gamma, seed, graph=False):
    B, P = eng.max_slots, 70
    tok = synth.make_tokens(B, P + 1, cfg["vocab"], seed)
    slots = i32(np.arange(B)[::-1].copy())
    eng.prefill(slots, tok[:, :P].cuda().contiguous())
    bufs = sdrl.SDBuffers(eng, B, gamma)
    last = tok[:, P].cuda().contiguous()
    got, g = [], None
    for it in range(n_steps):
        if graph and it:
            if g is None:
                torch.cuda.synchronize()
                g = sdrl.StepGraph(eng, bufs, slots, last, 1.0, seed, 3)
            g.replay()
            torch.ones(1000, device="cuda").sum().item()
        else:
            sdrl.sd_step(eng, bufs, slots, last, 1.0, seed, 3)
            last.copy_(bufs.next_tok)
        eng.sync()
        got.append({n: getattr(bufs, n).clone() for n in ("draft_tok", "q_logits", "p_logits", "out_tok", "n_emit")})
    return got


def same(a, b):
    for it, (x, y) in enumerate(zip(a, b)):
        for n in x:
            assert torch.equal(x[n], y[n]), (it, n)


def test_page_order_graph_and_poison_change_nothing():
    say("kv4 engine: pages, graph, poison")
    cfg, gamma, seed = GQA, 3, 8
    W = [w.cuda() for w in synth.make_weights(cfg, seed, "cpu", std=0.05)]
    base = None
    for kw, graph, poison in ((dict(order=False), False, False), (dict(page=64, seed=3), False, False), (dict(page=96), True, False),
                              (dict(seed=5), False, True)):
        eng, cache = setup(cfg, W, 4, 128, gamma, **kw)
        eng.set_debug(poison=poison)
        got = run_steps(eng, cache, cfg, 4, gamma, seed, graph)
        if base is None:
            base = got
        same(base, got)
        if poison:                                             # the rows past each length are NaN groups
            n = cache.kv_len.cpu().tolist()
            ko = torch.zeros((4, 2, cfg["n_kv"], cfg["head_dim"]), dtype=torch.bfloat16, device="cuda")
            vo = torch.zeros_like(ko)
            sdrl.kv4_read(cache, 1, i32([0, 1, 2, 3]), i32([x - 1 for x in n]), ko, vo)
            cache.check()
            assert torch.isfinite(ko[:, 0]).all() and torch.isfinite(vo[:, 0]).all()
            assert torch.isnan(ko[:, 1]).all() and torch.isnan(vo[:, 1]).all()
        eng.close()


def test_long_prefill_takes_its_own_workspace_and_equals_short_rounds():
    """Prefill of more rows than a step's (its own workspace, allocated before or after the binding) against the same
    prompt in pieces: layer 0's rows do not depend on the rounds."""
    say("kv4 long prefill")
    cfg, seed = MHA, 9
    W = [w.cuda() for w in synth.make_weights(cfg, seed, "cpu", std=0.05)]
    tok = synth.make_tokens(2, 600, cfg["vocab"], seed).cuda()
    slots, pools = i32([0, 1]), []
    for mode in ("whole", "pieces", "after dense"):
        if mode == "after dense":
            eng, k, v, n = make_engine(cfg, W, 2, 704, 2)
            eng.prefill(slots, tok)
            cache = eng.alloc_kv4(44, 32, torch.arange(44, dtype=torch.int32, device="cuda").reshape(2, 22))
            eng.bind_kv4(cache)
        else:
            eng, cache = setup(cfg, W, 2, 704, 2, order=False)
        if mode == "pieces":
            for t in range(0, 600, 200):
                eng.prefill(slots, tok[:, t:t + 200].contiguous())
        else:
            eng.prefill(slots, tok)
        eng.sync()
        assert cache.kv_len.tolist() == [600, 600]
        pools.append(cache.pages[:44, 0].clone())
        eng.close()
    assert torch.equal(pools[0], pools[2])
    a, b = (p.view(torch.int32) for p in (pools[0], pools[1]))
    assert (a != b).float().mean().item() < 0.01                 # GEMMs of other heights sum in another order


def test_bindings_replace_each_other():
    """A dense cache bound after a 4-bit one gives what it gives alone."""
    say("kv4 then dense")
    cfg, gamma, seed = GQA, 2, 11
    W = [w.cuda() for w in synth.make_weights(cfg, seed, "cpu")]
    outs = []
    for first in (False, True):
        eng, k, v, kv_len = make_engine(cfg, W, 2, 128, gamma)
        if first:
            cache = eng.alloc_kv4(8, 32, torch.arange(8, dtype=torch.int32, device="cuda").reshape(2, 4))
            eng.bind_kv4(cache)
            run_steps(eng, cache, cfg, 1, gamma, seed)
            eng.bind_kv(k, v, kv_len)
        outs.append(run_steps(eng, None, cfg, 2, gamma, seed))
        eng.close()
    same(*outs)


def test_set_rope_reaches_the_dense_cache():
    """The unscaled table set by hand is the engine's own; a scaled one moves the logits."""
    say("set_rope")
    cfg, gamma, seed = GQA, 2, 13
    W = [w.cuda() for w in synth.make_weights(cfg, seed, "cpu", std=0.05)]
    outs = []
    for rope in (None, sdrl.RopeConfig(cfg["rope_theta"], 128), sdrl.RopeConfig(cfg["rope_theta"], 128, "linear", 4.0)):
        eng, k, v, kv_len = make_engine(cfg, W, 2, 128, gamma)
        if rope is not None:
            eng.set_rope(rope)
        outs.append(run_steps(eng, None, cfg, 2, gamma, seed))
        eng.close()
    assert torch.equal(outs[0][0]["out_tok"], outs[1][0]["out_tok"])
    d = (outs[0][0]["p_logits"] - outs[1][0]["p_logits"]).abs().max().item()
    top = outs[0][0]["p_logits"].abs().max().item()
    assert d <= 2e-2 * top and (outs[0][0]["p_logits"] - outs[2][0]["p_logits"]).abs().max().item() > 2e-2 * top
    with pytest.raises(sdrl.SDError, match="head_dim"):
        eng2, *_ = make_engine(cfg, W, 2, 128, gamma)
        eng2.set_rope(sdrl.RopeConfig(1e4, 64))


def test_device_errors_and_refusals():
    say("kv4 engine errors")
    cfg, gamma = GQA, 2
    W = [w.cuda() for w in synth.make_weights(cfg, 1, "cpu")]
    eng, cache = setup(cfg, W, 2, 128, gamma)
    cache.kv_len.fill_(100)
    keep = cache.block_table.clone()
    cache.block_table[1, 1] = 99
    bufs = sdrl.SDBuffers(eng, 2, gamma)
    eng.draft(i32([0, 1]), i32([1, 2]), gamma, 1.0, 1, 1, bufs.draft_tok, bufs.q_logits, bufs.q_stats)
    with pytest.raises(sdrl.SDError, match="block-table"):
        eng.sync()
    cache.block_table.copy_(keep)
    cache.kv_len.fill_(127)
    eng.draft(i32([0, 1]), i32([1, 2]), gamma, 1.0, 1, 1, bufs.draft_tok, bufs.q_logits, bufs.q_stats)
    with pytest.raises(sdrl.SDError, match="max_ctx"):
        eng.sync()
    eng.draft(i32([0, 7]), i32([1, 2]), gamma, 1.0, 1, 1, bufs.draft_tok, bufs.q_logits, bufs.q_stats)
    with pytest.raises(sdrl.SDError, match="slot"):
        eng.sync()
    eng.sync()
    L = sdrl.lib()
    for name, val in (("n_layers", 1), ("n_kv", 1), ("head_dim", 64), ("max_slots", 1), ("max_ctx", 96), ("n_pages", 0),
                      ("page_size", 40), ("pages", None)):
        c = sdrl.KV4Struct.from_buffer_copy(cache.c)
        setattr(c, name, val)
        assert L.sd_bind_kv4(eng.h, C.byref(c)) == sdrl.SD_E_INVAL, name
    eng.close()
    wide = sdrl.Engine(MHA, 2048, 1 << 20, 1)
    c = sdrl.KV4Struct.from_buffer_copy(cache.c)
    c.n_layers, c.n_kv, c.head_dim = MHA["n_layers"], MHA["n_kv"], MHA["head_dim"]
    c.max_slots, c.max_ctx, c.pages_per_seq = 2048, 1 << 20, 1 << 15
    assert L.sd_bind_kv4(wide.h, C.byref(c)) == sdrl.SD_E_UNSUPPORTED  # positions past 31 bits in all
    wide.close()
    f32, *_ = make_engine(synth.TINY, [w.cuda() for w in synth.make_weights(synth.TINY, 1, "cpu")], 2, 64, 2)
    c = sdrl.kv4_pages(8, 2, 4, 64, 32)
    cache = sdrl.KV4Cache(c, torch.zeros((2, 2), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), 64)
    with pytest.raises(sdrl.SDError, match="bf16"):
        f32.bind_kv4(cache)
    f32.close()
