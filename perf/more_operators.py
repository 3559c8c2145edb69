"""Cases of the operators of grouped rollouts: several responses are sampled of each prompt and learned from.

  append     new rows of keys and values, rotated and stored in bf16 pages, with their queries
  attention  a batch whose groups share a prompt's pages: the shared positions are read once for a group
  logp       log-probabilities and entropy of tokens from logits rows, with or without the gradient
  policy     the clipped policy loss with a KL term, an entropy term and a filter by importance ratio, with the
             gradient of the logits
"""
import math

import torch

own = False

LAYERS, LAYER = 2, 1                # the cases run on the second of two layers: a layer has its own offset in a page


# ------------------------------------------------------------------ cases
def _append(name, B, n, base, n_q, n_kv, D, rot, layout, page, ragged, dtype="bf16"):
    return dict(name=name, op="append", B=B, n=n, base=base, n_q=n_q, n_kv=n_kv, D=D, rot=rot, layout=layout,
                page=page, ragged=ragged, dtype=dtype)


def _attention(name, groups, size, n, prefix, tail, n_q, n_kv, D, page, ragged):
    """groups of `size` sequences sharing `prefix` positions, with up to `tail` of their own, the n new rows among them."""
    return dict(name=name, op="attention", groups=groups, size=size, n=n, prefix=prefix, tail=tail, n_q=n_q, n_kv=n_kv,
                D=D, page=page, ragged=ragged)


def _logp(name, rows, V, dtype, T, grad):
    return dict(name=name, op="logp", rows=rows, V=V, dtype=dtype, T=T, grad=grad)


def _policy(name, rows, V, dtype, T, kl, entropy, pad):
    """pad: the share of rows whose token is padding (weight 0)."""
    return dict(name=name, op="policy", rows=rows, V=V, dtype=dtype, T=T, kl=kl, entropy=entropy, pad=pad)


def listed():
    return [
        # one group's decode step on the 8B shape: latency
        _append("append_b8_n1_8b", 8, 1, 700, 32, 8, 128, 128, "half", 64, False),
        # a prefill of ragged prompts, fp32 rows, pairs interleaved, half of a small head rotated
        _append("append_b24_n509_f32", 24, 509, 33, 8, 2, 64, 32, "interleaved", 32, True, "f32"),
        # decode of a single group of 8 behind a prompt of 512: latency
        _attention("attn_1x8_n1_512", 1, 8, 1, 512, 200, 32, 8, 128, 64, False),
        # decode of 8 groups of 8 behind prompts of 2048 on the 8B shape, responses of different lengths
        _attention("attn_8x8_n1_2048", 8, 8, 1, 2048, 512, 32, 8, 128, 64, True),
        # groups of five, verify blocks of 3 of which some rows are missing, an odd prompt, small heads, small pages
        _attention("attn_5x5_n3_ragged_d64", 5, 5, 3, 777, 300, 8, 2, 64, 32, True),
        # the verify block, gamma 4, of 8 groups of 8 at 8192 positions on the 32B shape
        _attention("attn_8x8_n5_8192_32b", 8, 8, 5, 8192, 600, 40, 8, 128, 64, False),
        # 64 sequences behind one long context
        _attention("attn_1x64_n1_32768", 1, 64, 1, 32768, 256, 32, 8, 128, 64, False),
        # log-probabilities of a decode step's tokens from the engine's logits: few long rows
        _logp("logp_64x128256_f32", 64, 128256, "f32", 1.0, False),
        # scoring of a batch of responses with the gradient, on the 32B shape's vocabulary
        _logp("logp_grad_2048x152064", 2048, 152064, "bf16", 1.0, True),
        # a small update on a tiny vocabulary: latency
        _policy("policy_96x512_f32", 96, 512, "f32", 1.0, 0.001, 0.0, 0.25),
        # fp32 logits, an odd vocabulary whose rows lie at any alignment, temperature and entropy term
        _policy("policy_1023x50257_f32", 1023, 50257, "f32", 0.7, 0.001, 0.01, 0.1),
        # an update's micro-batch on the 8B shape's vocabulary, with padding
        _policy("policy_8192x128256", 8192, 128256, "bf16", 1.0, 0.001, 0.0, 0.2),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(("append", "attention", "attention", "attention", "logp", "policy", "policy"))
    if op in ("append", "attention"):
        n_q, n_kv, D = rng.choice(((32, 8, 128), (40, 8, 128), (4, 4, 64), (4, 2, 128), (8, 2, 64), (16, 1, 128),
                                   (28, 4, 128)))
        page, ragged = rng.choice((32, 64, 96, 128)), rng.random() < 0.5
        if op == "append":
            B = _log_int(rng, 1, 64)
            c = _append("", B, _log_int(rng, 1, 12000 // B), rng.randint(0, 4000), n_q, n_kv, D, 16 * rng.randint(0, D // 16),
                        rng.choice(("half", "interleaved")), page, ragged, rng.choice(("bf16", "bf16", "f32")))
        else:
            groups, size = _log_int(rng, 1, 8), _log_int(rng, 1, 64)
            size = min(size, 64 // groups)
            n = rng.choice((1, 1, rng.randint(2, 12)))
            tail = n + _log_int(rng, 1, 600)
            most = min(32768, 550_000 // (groups * size), 2_400_000 // (groups * size * n))
            c = _attention("", groups, size, n, rng.choice((0,) + 9 * (_log_int(rng, 17, max(most, 18)),)), tail, n_q, n_kv, D,
                           page, ragged)
    else:
        V = rng.choice((512, 32000, 50257, 128256, 152064, _log_int(rng, 100, 200000)))
        rows = _log_int(rng, 1, min(20000, 500_000_000 // V))
        dtype, T = rng.choice(("f32", "bf16")), rng.choice((1.0, 1.0, 0.6, 1.3))
        if op == "logp":
            c = _logp("", rows, V, dtype, T, rng.random() < 0.5)
        else:
            c = _policy("", rows, V, dtype, T, rng.choice((0.0, 0.001, 0.05)), rng.choice((0.0, 0.01)), rng.choice((0.0, 0.2, 0.5)))
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _i32(values, device="cuda"):
    return torch.tensor(values, dtype=torch.int32, device=device)


def _table(max_ctx, rot):
    ang = torch.arange(max_ctx, dtype=torch.float64, device="cuda")[:, None] * torch.pow(
        torch.tensor(5e5, dtype=torch.float64, device="cuda"),
        -torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / max(rot, 1))
    return torch.stack((ang.cos(), ang.sin()), -1).float()


def _pools(case, n_pages, gd):
    shape = (n_pages, LAYERS, case["n_kv"], case["page"], case["D"])
    k, v = (torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    step = max(1, (1 << 26) // k[0, LAYER].numel())
    for p0 in range(0, n_pages, step):
        for t in (k, v):
            blk = t[p0:p0 + step, LAYER]
            blk.copy_(torch.randn(blk.shape, generator=gd, device="cuda"))
    return k, v


def _prepare_append(case, g, gd):
    B, n, n_q, n_kv, D = (case[k] for k in ("B", "n", "n_q", "n_kv", "D"))
    u = torch.rand((2, B), generator=g)
    base, lens = [case["base"]] * B, [n] * B
    if case["ragged"]:
        base = (case["base"] * (0.1 + 0.9 * u[0])).int().tolist()
        lens = ((n + 1) * u[1]).int().tolist()                     # some sequences have no row at all
        lens[0] = n
    max_ctx = max(base) + n
    per = -(-max_ctx // case["page"])
    n_pages = B * per + 3
    table = torch.randperm(n_pages, generator=g)[:B * per].to(torch.int32).reshape(B, per).cuda()
    shape = (n_pages, LAYERS, n_kv, case["page"], D)
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    # the rows as a projection gives them: q, k and v side by side
    qkv = torch.randn((B, n, n_q + 2 * n_kv, D), generator=gd, device="cuda").to(dtype)
    return dict(case, k_pages=torch.zeros(shape, dtype=torch.bfloat16, device="cuda"),
                v_pages=torch.zeros(shape, dtype=torch.bfloat16, device="cuda"), block_table=table, max_ctx=max_ctx,
                kv_len=_i32(base), slots=_i32(list(range(B))), lens=_i32(lens) if case["ragged"] else None,
                q=qkv[:, :, :n_q], k=qkv[:, :, n_q:n_q + n_kv], v=qkv[:, :, n_q + n_kv:], table=_table(max_ctx, case["rot"]),
                q_out=torch.zeros((B, n, n_q, D), dtype=torch.bfloat16, device="cuda"))


def _prepare_attention(case, g, gd):
    G, size, n, P, page = (case[k] for k in ("groups", "size", "n", "prefix", "page"))
    B = G * size
    u = torch.rand((2, B), generator=g)
    own_len, lens = [case["tail"] - n] * B, [n] * B
    if case["ragged"]:
        own_len = ((case["tail"] - n) * u[0]).int().tolist()
        lens = [max(1, x) for x in ((n + 1) * u[1]).int().tolist()]
        if B > 2:
            lens[B // 2] = 0                                       # a sequence without a row
    base = [P + x for x in own_len]
    max_ctx = P + case["tail"]
    per = -(-max_ctx // page)
    shared = P // page                                             # whole pages of the prompt; its rest is copied
    n_pages = G * shared + B * (per - shared) + 3
    pages = torch.randperm(n_pages, generator=g).to(torch.int32)
    # slots in any order, the members of a group next to each other in the batch
    slots = torch.randperm(B + 2, generator=g)[:B]
    table = torch.full((B + 2, per), -1, dtype=torch.int32)
    front = pages[:G * shared].reshape(G, 1, shared).expand(G, size, shared).reshape(B, shared)
    back = pages[G * shared:G * shared + B * (per - shared)].reshape(B, per - shared)
    table[slots] = torch.cat((front, back), 1)
    group, kv_len = torch.full((B + 2,), -1, dtype=torch.int32), torch.zeros(B + 2, dtype=torch.int32)
    group[slots] = torch.arange(B, dtype=torch.int32) // size
    kv_len[slots] = torch.tensor(base, dtype=torch.int32)
    k, v = _pools(case, n_pages, gd)
    rest = P % page
    if rest:                                                       # each member's copy of the prompt's last positions
        own_pg = back[:, 0].long().reshape(G, size)
        for t in (k, v):
            t[own_pg.flatten().cuda(), LAYER, :, :rest] = t[own_pg[:, :1].expand(G, size).flatten().cuda(), LAYER, :, :rest]
    q = torch.randn((B, n, case["n_q"], case["D"]), generator=gd, device="cuda").bfloat16()
    return dict(case, k_pages=k, v_pages=v, block_table=table.cuda(), kv_len=kv_len.cuda(), slots=slots.int().cuda(),
                group=group.cuda(), length=_i32([P] * G), max_ctx=max_ctx, lens=_i32(lens) if case["ragged"] else None, q=q,
                out=torch.zeros_like(q))


def _prepare_rows(case, g, gd):
    rows, V, T = case["rows"], case["V"], case["T"]
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    logits = torch.empty((rows, V), dtype=dtype, device="cuda")
    tokens = torch.empty(rows, dtype=torch.int32, device="cuda")
    logp = torch.empty(rows, dtype=torch.float32, device="cuda")
    step = max(1, (1 << 28) // V)
    for r0 in range(0, rows, step):                                # a few likely tokens in a row, the rest far below
        x = torch.randn((min(step, rows - r0), V), generator=gd, device="cuda") * 2
        x[:, :8] += 6 * torch.rand((x.shape[0], 8), generator=gd, device="cuda") + 6
        x = x.roll(int(torch.randint(0, V, (1,), generator=g)), 1)
        logits[r0:r0 + step] = x
        x = logits[r0:r0 + step].float() / T
        u = torch.empty_like(x).exponential_(generator=gd)
        t = (x - u.log()).argmax(1)                                # drawn from the softmax
        del u
        tokens[r0:r0 + step] = t.int()
        logp[r0:r0 + step] = (x.gather(1, t[:, None])[:, 0] - torch.logsumexp(x, 1)).float()
        del x
    st = dict(case, logits=logits, tokens=tokens)
    if case["op"] == "logp":
        if case["grad"]:
            st["dlogp"] = torch.randn(rows, generator=gd, device="cuda") / rows
            st["dentropy"] = 0.01 * torch.randn(rows, generator=gd, device="cuda") / rows
            st["dlogits"] = torch.empty_like(logits)
        return st
    def noise(width, *borders):
        """Steps of a policy's log-probabilities; those next to a border of the loss are moved off it."""
        d = width * torch.randn(rows, generator=gd, device="cuda")
        for b in borders:
            d = torch.where((d - b).abs() < 2e-3, d + 6e-3, d)
        return d
    # the policy after a few updates, the one that the rollout ran with, and the reference
    st["old"] = logp - noise(0.15, math.log(0.8), math.log(1.28))
    st["behavior"] = st["old"] - noise(0.3, math.log(0.5), math.log(2.0))
    st["ref"] = logp - noise(0.3)
    st["advantage"] = torch.randn(rows, generator=gd, device="cuda")
    live = torch.rand(rows, generator=gd, device="cuda") >= case["pad"]
    live[0] = True
    st["weight"] = live.float() / live.sum()
    st["dlogits"] = torch.empty_like(logits)
    return st


def prepare(case, seed):
    g = torch.Generator().manual_seed(seed)
    gd = torch.Generator(device="cuda").manual_seed(seed)
    return dict(append=_prepare_append, attention=_prepare_attention, logp=_prepare_rows, policy=_prepare_rows)[case["op"]](case, g, gd)


CLIP_LOW, CLIP_HIGH, IS_LOW, IS_HIGH = 0.2, 0.28, 0.5, 2.0


# ------------------------------------------------------------------ plain forms
def _rotate(x, table, pos, rot, layout):
    """x [B, n, heads, D] rotated at pos [B, n], rounded to bf16: products in 64 bits, where a rounding is decided."""
    cs = table[pos].double()[:, :, None]                        # [B, n, 1, rot / 2, 2]
    c, s = cs[..., 0], cs[..., 1]
    x = x.double()
    if layout == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat((a * c - b * s, a * s + b * c, x[..., rot:]), -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.cat((torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2), x[..., rot:]), -1)
    return y.bfloat16()


def _plain_append(st):
    B, n, page = st["B"], st["n"], st["page"]
    i = torch.arange(n, device="cuda")
    pos = st["kv_len"].long()[:, None] + i
    live = i[None] < st["lens"][:, None] if st["lens"] is not None else torch.ones_like(pos, dtype=torch.bool)
    q, k = (_rotate(st[x], st["table"], pos, st["rot"], st["layout"]) for x in ("q", "k"))
    q = q.masked_fill(~live[..., None, None], 0)
    at = st["block_table"].long().gather(1, pos // page)[live], (pos % page)[live]
    st["k_pages"][at[0], LAYER, :, at[1]] = k[live]
    st["v_pages"][at[0], LAYER, :, at[1]] = st["v"].bfloat16()[live]
    return q, st["k_pages"][:, LAYER], st["v_pages"][:, LAYER]


def _cached(st, name):
    """Keys or values [B, n_kv, positions, D] in 32 bits, gathered from the pages."""
    x = st[name][:, LAYER][st["block_table"].long()[st["slots"].long()]]       # [B, pages, H, page, D]
    return x.transpose(1, 2).flatten(2, 3).float()


def _plain_attention(st):
    B, n, H, D = st["groups"] * st["size"], st["n"], st["n_kv"], st["D"]
    G = st["n_q"] // H
    k, v = _cached(st, "k_pages"), _cached(st, "v_pages")
    p = torch.arange(k.shape[2], device="cuda")
    i = torch.arange(n, device="cuda")
    last = st["kv_len"][st["slots"].long()][:, None] + i                       # [B, n]
    q = st["q"].float().reshape(B, n, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * n, D)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(D)
    seen = (p <= last[..., None])[:, None].repeat(1, 1, G, 1)                  # [B, 1, G n, positions]
    s = s.masked_fill(~seen, float("-inf"))
    e = torch.exp(s - s.amax(-1, keepdim=True))
    o = torch.matmul(e, v.masked_fill((p > last[:, -1:])[:, None, :, None], 0.0)) / e.sum(-1, keepdim=True)
    o = o.reshape(B, H, G, n, D).permute(0, 3, 1, 2, 4).reshape(B, n, st["n_q"], D).bfloat16()
    if st["lens"] is None:
        return o
    return torch.where((i[None] < st["lens"][:, None])[..., None, None], o, torch.zeros_like(o))


def _softmax_parts(st):
    """x = logits / T less the row's maximum, e^x, its sum and that one's logarithm, the tokens' log-probabilities, the
    entropy, and the rows' norm: (largest logit, ln sum e^x)."""
    x = st["logits"].float() / st["T"]
    top = x.amax(1, keepdim=True)
    x = x - top
    e = torch.exp(x)
    total = e.sum(1, keepdim=True)
    z = torch.log(total)
    logp = (x.gather(1, st["tokens"].long()[:, None]) - z)[:, 0]
    entropy = (z - (e * x).sum(1, keepdim=True) / total)[:, 0]
    return x, e, total, z, logp, entropy, torch.stack((st["logits"].amax(1).float(), z[:, 0]), 1)


def _logits_gradient(st, x, e, total, z, entropy, dlogp, dentropy):
    p = e / total
    d = -dlogp[:, None] * p
    if dentropy is not None:
        d -= dentropy[:, None] * p * (x - z + entropy[:, None])
    d.scatter_add_(1, st["tokens"].long()[:, None], dlogp[:, None])
    return (d / st["T"]).to(st["logits"].dtype)


def _plain_logp(st):
    x, e, total, z, logp, entropy, norm = _softmax_parts(st)
    if not st["grad"]:
        return logp, entropy, norm
    return logp, entropy, norm, _logits_gradient(st, x, e, total, z, entropy, st["dlogp"], st["dentropy"])


def _plain_policy(st):
    x, e, total, z, logp, entropy, _ = _softmax_parts(st)
    A = st["advantage"]
    far = st["old"] - st["behavior"]
    on = st["weight"] != 0
    kept = on & (far >= math.log(IS_LOW)) & (far <= math.log(IS_HIGH))
    w = torch.where(kept, st["weight"], 0.0)
    r = torch.exp(logp - st["old"])
    free, cut = r * A, r.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * A
    clipped = cut < free
    gap = st["ref"] - logp
    kl = torch.exp(gap) - gap - 1
    pg = -torch.minimum(free, cut)
    dlogp = w * (torch.where(clipped, 0.0, -free) + st["kl"] * (1 - torch.exp(gap)))
    stats = torch.stack([(w * (pg + st["kl"] * kl - st["entropy"] * entropy)).sum(), (w * pg).sum(), (w * kl).sum(),
                         (w * entropy).sum(), (w * clipped).sum(), (st["weight"] * (on & ~kept)).sum()])
    d = _logits_gradient(st, x, e, total, z, entropy, dlogp, -st["entropy"] * w)
    return stats, torch.where(kept, logp, 0.0), torch.where(kept, entropy, 0.0), d


# ------------------------------------------------------------------ the framework's calls
def _handle(st):
    """The description of the cache's tensors and the loss, made once as a user's program does, and the workspace."""
    if "cache" not in st:
        from paper_2606_18967_amd import sdrl
        st["sdrl"] = sdrl
        if st["op"] in ("append", "attention"):
            st["cache"] = sdrl.KVPages(st["k_pages"], st["v_pages"], st["block_table"], st["kv_len"], st["max_ctx"])
        if st["op"] == "attention":
            st["groups_"] = sdrl.PrefixGroups(st["group"], st["length"])
            size = sdrl.prefix_workspace_bytes(st["cache"], st["groups"] * st["size"], st["n"], st["n_q"])
            st["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        elif st["op"] != "append":
            size = sdrl.logits_workspace_bytes(st["rows"], st["V"])
            st["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
            st["cache"] = None
            if st["op"] == "policy":
                st["cache"] = sdrl.PolicyLoss(clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=st["kl"], entropy_coef=st["entropy"],
                                              is_low=IS_LOW, is_high=IS_HIGH, temperature=st["T"])
    return st["sdrl"], st["cache"]


def run(state):
    st = state
    if own:
        sdrl, cache = _handle(st)
        if st["op"] == "append":
            sdrl.kv_append(cache, LAYER, st["slots"], st["k"], st["v"], st["q"], st["q_out"], rope=st["table"],
                           layout=st["layout"], lens=st["lens"])
            return st["q_out"], st["k_pages"][:, LAYER], st["v_pages"][:, LAYER]
        if st["op"] == "attention":
            return sdrl.prefix_attention(cache, st["groups_"], LAYER, st["slots"], st["q"], st["out"], lens=st["lens"],
                                         workspace=st["workspace"])
        if st["op"] == "logp":
            logp, entropy, norm = sdrl.token_logprobs(st["logits"], st["tokens"], st["T"], workspace=st["workspace"])
            if not st["grad"]:
                return logp, entropy, norm
            return logp, entropy, norm, sdrl.token_logprobs_grad(st["logits"], st["tokens"], norm, st["dlogp"], st["T"], entropy=entropy,
                                                                 dentropy=st["dentropy"], out=st["dlogits"])
        out = sdrl.policy_loss(cache, st["logits"], st["tokens"], st["old"], st["advantage"], st["weight"], ref_logp=st["ref"],
                               behavior_logp=st["behavior"], dlogits=st["dlogits"], workspace=st["workspace"])
        return out.stats, out.logp, out.entropy, out.dlogits
    return dict(append=_plain_append, attention=_plain_attention, logp=_plain_logp, policy=_plain_policy)[st["op"]](st)


# ------------------------------------------------------------------ work
def work(case):
    if case["op"] in ("append", "attention"):
        n, n_q, n_kv, D = (case[k] for k in ("n", "n_q", "n_kv", "D"))
    if case["op"] == "append":
        rows = case["B"] * n * (0.5 if case["ragged"] else 1.0)
        el = 4 if case["dtype"] == "f32" else 2
        return dict(bytes=rows * (n_q + 2 * n_kv) * D * (el + 2) + n * case["rot"] * 4, flops=rows * (n_q + n_kv) * D * 3)
    if case["op"] == "attention":
        B, share = case["groups"] * case["size"], 0.5 if case["ragged"] else 1.0
        tail, rows = (case["tail"] - n) * share + n, B * n * (0.75 if case["ragged"] and n > 1 else 1.0)
        return dict(bytes=(case["groups"] * case["prefix"] + B * tail) * n_kv * D * 4 + rows * n_q * D * 4,
                    flops=4.0 * rows * (case["prefix"] + tail) * n_q * D)
    cells, el = case["rows"] * case["V"], 4 if case["dtype"] == "f32" else 2
    if case["op"] == "logp":
        return dict(bytes=cells * el * (2 if case["grad"] else 1) + case["rows"] * 16, flops=cells * (10 if case["grad"] else 5))
    live = 1 - case["pad"]
    return dict(bytes=cells * el * (1 + live) + case["rows"] * 32, flops=cells * live * 10)


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_append(st):
    """Sequence by sequence, with the rotation as a product of complex numbers."""
    rot, n, page = st["rot"], st["n"], st["page"]
    q_out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    pools = [torch.zeros_like(st[x][:, LAYER], dtype=torch.float64) for x in ("k_pages", "v_pages")]
    first = torch.arange(rot // 2, device="cuda") * (1 if st["layout"] == "half" else 2)
    second = first + (rot // 2 if st["layout"] == "half" else 1)
    for b in range(st["B"]):
        m = int(st["lens"][b]) if st["lens"] is not None else n
        base = int(st["kv_len"][b])
        turn = torch.view_as_complex(st["table"][base:base + m].double().contiguous())[:, None]
        rows = []
        for name in ("q", "k", "v"):
            x = st[name][b, :m].double().clone()
            if name != "v" and rot:
                z = torch.complex(x[..., first], x[..., second]) * turn
                x[..., first], x[..., second] = z.real, z.imag
            rows.append(x)
        q_out[b, :m] = rows[0]
        P = torch.arange(base, base + m, device="cuda")
        pg = st["block_table"][b].long()[P // page]
        for pool, x in zip(pools, rows[1:]):
            pool[pg, :, P % page] = x
    return q_out, pools[0], pools[1]


def _exact_attention(st):
    """Sequence by sequence and head by head."""
    H, n, page, D = st["n_kv"], st["n"], st["page"], st["D"]
    G = st["n_q"] // H
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for b in range(st["groups"] * st["size"]):
        slot = int(st["slots"][b])
        m, base = int(st["lens"][b]) if st["lens"] is not None else n, int(st["kv_len"][slot])
        if m == 0:
            continue
        P = torch.arange(base + m, device="cuda")
        pg = st["block_table"][slot].long()[P // page]
        seen = P[None] <= base + torch.arange(m, device="cuda")[:, None]
        for h in range(H):
            k, v = (st[x][pg, LAYER, h, P % page].double() for x in ("k_pages", "v_pages"))
            q = st["q"][b, :m, h * G:(h + 1) * G].double()                     # [m, G, D]
            s = torch.matmul(q.reshape(m * G, D), k.t().contiguous()).reshape(m, G, -1) * D ** -0.5
            a = torch.softmax(torch.where(seen[:, None], s, -math.inf), dim=-1)
            out[b, :m, h * G:(h + 1) * G] = torch.matmul(a.reshape(m * G, -1), v).reshape(m, G, D)
    return out


def _exact_rows(st):
    """Row blocks, by torch's own softmax in 64 bits."""
    rows, V, T = st["rows"], st["V"], st["T"]
    policy = st["op"] == "policy"
    logp, entropy = (torch.zeros(rows, dtype=torch.float64, device="cuda") for _ in range(2))
    norm = torch.zeros((rows, 2), dtype=torch.float64, device="cuda")
    grad = torch.zeros((rows, V), dtype=torch.float32, device="cuda") if policy or st["grad"] else None
    sums = torch.zeros(6, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 26) // V)
    for r0 in range(0, rows, step):
        cut = slice(r0, min(r0 + step, rows))
        y = torch.log_softmax(st["logits"][cut].double() / T, 1)
        p = torch.exp(y)
        at = st["tokens"][cut].long()[:, None]
        lp = y.gather(1, at)[:, 0]
        H = -torch.where(p > 0, p * y, 0.0).sum(1)
        norm[cut, 0] = st["logits"][cut].double().max(1)[0]
        norm[cut, 1] = -y.max(1)[0]
        if policy:
            w, old, A = st["weight"][cut].double(), st["old"][cut].double(), st["advantage"][cut].double()
            ratio_b = torch.exp(old - st["behavior"][cut].double())
            ok = (w != 0) & (ratio_b >= IS_LOW) & (ratio_b <= IS_HIGH)
            sums[5] += w[~ok].sum()
            w = w * ok
            r = torch.exp(lp - old)
            over = ((A > 0) & (r > 1 + CLIP_HIGH)) | ((A < 0) & (r < 1 - CLIP_LOW))
            surrogate = A * torch.where(over, torch.where(A > 0, 1.0 + CLIP_HIGH, 1.0 - CLIP_LOW), r)
            back = st["ref"][cut].double() - lp
            kl = torch.expm1(back) - back
            sums[:5] += torch.stack([(w * (st["kl"] * kl - surrogate - st["entropy"] * H)).sum(), -(w * surrogate).sum(), (w * kl).sum(),
                                     (w * H).sum(), (w * over).sum()])
            gl = -w * (torch.where(over, 0.0, A * r) + st["kl"] * torch.expm1(back))
            gh = -st["entropy"] * w
            lp, H = lp * ok, H * ok
        elif grad is not None:
            gl, gh = st["dlogp"][cut].double(), st["dentropy"][cut].double()
        logp[cut], entropy[cut] = lp, H
        if grad is not None:
            H = -torch.where(p > 0, p * y, 0.0).sum(1, keepdim=True)
            d = -gl[:, None] * p - gh[:, None] * torch.where(p > 0, p * (y + H), 0.0)
            d[torch.arange(d.shape[0], device="cuda"), at[:, 0]] += gl
            grad[cut] = (d / T).float()
    if policy:
        return sums, logp, entropy, grad
    return (logp, entropy, norm) if grad is None else (logp, entropy, norm, grad)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(st)
    return _exact_attention(st) if case["op"] == "attention" else _exact_rows(st)
