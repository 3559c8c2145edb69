"""The 4-bit KV cache's operators against plain 64-bit implementations (kv4_ref): the rotary table, the append
(bytes of the whole pool), the read-back and the attention, over head layouts, odd lengths and places, strides,
masks, values that are not finite, streams, graphs and pools past 4 GB."""
import numpy as np
import pytest
import torch

import kv4_ref as ref
from paper_2606_18967_amd import sdrl

from gpu_common import i32, say

pytestmark = pytest.mark.gpu


def make_cache(n_layers, n_kv, D, slots, max_ctx, page, seed, spare=2, random_pool=True):
    g = torch.Generator().manual_seed(seed)
    per = -(-max_ctx // page)
    n_pages = slots * per + spare
    pages = sdrl.kv4_pages(n_pages, n_layers, n_kv, D, page)
    if random_pool:
        pages.copy_(torch.randint(0, 256, pages.shape, generator=g, dtype=torch.uint8))
    table = torch.randperm(n_pages, generator=g)[:slots * per].to(torch.int32).reshape(slots, per).cuda()
    return sdrl.KV4Cache(pages, table, torch.zeros(slots, dtype=torch.int32, device="cuda"), max_ctx)


def host(cache):
    return ref.HostCache(cache.pages.cpu().numpy(), cache.block_table.cpu().numpy(), cache.head_dim)


def same_pool(cache, hc):
    got = cache.pages.cpu().numpy().view(np.uint32).reshape(hc.w.shape)
    bad = np.argwhere(got != hc.w)
    assert not len(bad), (len(bad), bad[:4], [(hex(got[tuple(b)]), hex(hc.w[tuple(b)])) for b in bad[:4]])


ROPES = [("none", dict(theta=1e4)), ("linear", dict(theta=1e4, factor=4.0)),
         ("llama3", dict(theta=5e5, factor=8.0, low=1.0, high=4.0, orig=8192)),
         ("yarn", dict(theta=1e6, factor=4.0, low=1.0, high=32.0, orig=4096)),
         ("yarn", dict(theta=1e4, factor=2.0, low=1.0, high=32.0, orig=2048, attn_factor=0.75))]


@pytest.mark.parametrize("n_pos,rot", [(1, 2), (63, 64), (64, 128), (65, 16), (4099, 256), (131072, 34)])
@pytest.mark.parametrize("scaling,kw", ROPES, ids=lambda x: x if isinstance(x, str) else "")
def test_rope_table(n_pos, rot, scaling, kw):
    say("rope_table", n_pos, rot, scaling)
    f, mul = ref.frequencies(rot=rot, scaling=scaling, **kw)
    kw = dict(kw)
    cfg = sdrl.RopeConfig(kw.pop("theta"), rot, scaling, kw.pop("factor", 1.0), kw.pop("low", 0.0), kw.pop("high", 0.0),
                          kw.pop("orig", 0), kw.pop("attn_factor", 0.0))
    out = torch.full((n_pos + 1, rot // 2, 2), 7.0, device="cuda")
    got = sdrl.rope_table(cfg, n_pos, out[:n_pos])
    ang = np.arange(n_pos)[:, None] * f
    want = np.stack((np.cos(ang), np.sin(ang)), -1) * mul
    # one rounding to fp32 of values up to mul, and an angle up to 1.3e5 that is off by some 2^-52 of itself
    tol = mul * (2.0 ** -24 + 1e-9)
    assert np.abs(got.cpu().numpy().astype(np.float64) - want).max() <= tol
    assert bool((out[n_pos] == 7.0).all())


def append_case(D, n_q, n_kv, B, n, base, lens, rot, layout, dtype, page, seed, tweak=None, pad=0):
    """Runs one append on a pool of random bytes and checks every byte of it, q_out and the read-back."""
    max_ctx = max(base) + n + 3
    slots = np.random.default_rng(seed).permutation(B + 2)[:B]
    cache = make_cache(2, n_kv, D, B + 2, max_ctx, page, seed)
    kv_len = np.full(B + 2, 5, np.int32)
    kv_len[slots] = base
    cache.kv_len.copy_(i32(kv_len))
    hc = host(cache)
    g = torch.Generator().manual_seed(seed + 1)
    units = n_q + 2 * n_kv + pad
    x = torch.randn((B, n, units, D), generator=g)
    if tweak is not None:
        tweak(x[:, :, n_q:n_q + n_kv], x[:, :, n_q + n_kv:n_q + 2 * n_kv])
    x = x.to(dtype).cuda()
    q, k, v = x[:, :, :n_q], x[:, :, n_q:n_q + n_kv], x[:, :, n_q + n_kv:n_q + 2 * n_kv]
    table = sdrl.rope_table(sdrl.RopeConfig(1e4, rot), max_ctx) if rot else None
    q_out = torch.full((B, n, n_q, D), 9.0, dtype=torch.bfloat16, device="cuda")
    ll = None if lens is None else i32(lens)
    sdrl.kv4_append(cache, 1, i32(slots), k, v, q, q_out, rope=table, layout=layout, lens=ll)
    k_out = torch.full((B, n, n_kv, D), 9.0, dtype=torch.bfloat16, device="cuda")
    v_out = k_out.clone()
    sdrl.kv4_read(cache, 1, i32(slots), i32(base), k_out, v_out, lens=ll)
    cache.check()
    tab = table.cpu().numpy() if rot else None
    xq, xk, xv = (t.float().cpu().numpy() for t in (q, k, v))
    for b in range(B):
        m = n if lens is None else lens[b]
        pos = base[b] + np.arange(m)
        yk = ref.rotate(xk[b, :m], tab, pos[:, None], rot, layout)
        yq = ref.rotate(xq[b, :m], tab, pos[:, None], rot, layout)
        want_k, want_v = np.empty((m, n_kv, D)), np.empty((m, n_kv, D))
        for is_v, y, want in ((False, yk, want_k), (True, xv[b, :m], want_v)):
            c, s, z = ref.quantize(y)
            want[:] = z[..., None].astype(np.float64) + s[..., None].astype(np.float64) * (c - 8)
            for i in range(m):
                for h in range(n_kv):
                    hc.put(int(slots[b]), 1, h, int(pos[i]), is_v, c[i, h], s[i, h], z[i, h])
        got_q = q_out[b, :m].float().cpu().numpy().astype(np.float64)
        # fp32 rotation (three roundings of up to |x| sqrt(2)), then bf16
        assert (np.abs(got_q - yq) <= 2.0 ** -8 * np.abs(yq) + 2.0 ** -21 * np.abs(xq[b, :m]).max(initial=0.0)).all()
        for got, want in ((k_out[b, :m], want_k), (v_out[b, :m], want_v)):
            assert np.array_equal(got.float().cpu().numpy(), ref.bf16(want.astype(np.float32)), equal_nan=True)
        for t in (q_out, k_out, v_out):
            assert bool((t[b, m:] == 9.0).all())               # rows past the sequence's stay as they were
    same_pool(cache, hc)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D,n_q,n_kv,rot,layout", [(128, 32, 8, 128, "half"), (64, 4, 4, 64, "half"),
                                                   (128, 5, 1, 32, "interleaved"), (64, 6, 3, 48, "interleaved"),
                                                   (128, 4, 2, 112, "half"), (64, 2, 2, 0, "half"),
                                                   (128, 2, 1, 128, "interleaved")])
def test_append(D, n_q, n_kv, rot, layout, dtype):
    say("append", D, n_q, n_kv, rot, layout, dtype)
    append_case(D, n_q, n_kv, 3, 5, [0, 27, 61], None, rot, layout, dtype, 32, 11)
    append_case(D, n_q, n_kv, 4, 19, [1, 96, 33, 40], [19, 0, 7, 1], rot, layout, dtype, 64, 12, pad=1)


@pytest.mark.parametrize("base", range(9))
def test_append_one_row_at_each_place(base):
    say("append one row", base)
    append_case(128, 4, 2, 1, 1, [base], None, 128, "half", torch.bfloat16, 32, 20 + base)


def test_append_prefill_across_pages():
    say("append prefill")
    append_case(128, 8, 2, 2, 300, [0, 95], [300, 211], 128, "half", torch.bfloat16, 96, 31)


def test_append_rows_that_are_hard_to_quantize():
    """Zero, constant, huge, tiny, one-sided and tied rows, and rows with NaN or infinities."""
    say("append special rows")

    def tweak(k, v):
        for x in (k, v):
            x[0, 0] = 0
            x[0, 1] = 3.25
            x[0, 2] *= 1e38
            x[0, 3] *= 1e-38
            x[0, 4] = 100 + x[0, 4].abs()
            x[0, 5] = torch.arange(x.shape[-1]) % 31 * 0.5          # range 15: s = 1, every second value half way
            x[0, 6] = -(torch.arange(x.shape[-1]) % 31) * 0.25
            x[0, 7, 0, 3] = float("nan")
            x[0, 8, 0, 5] = float("inf")
            x[0, 9, 0, 7] = -float("inf")
            x[0, 10] = torch.tensor([-3e38, 3e38]).repeat(x.shape[-1] // 2)
            x[0, 11] = 1e-40
            x[0, 12] = 0
            x[0, 12, 0, 0] = 1e-40                                   # a step below the smallest number
    for dtype in (torch.bfloat16, torch.float32):
        append_case(128, 2, 1, 1, 14, [5], None, 0, "half", dtype, 32, 41, tweak)
        append_case(64, 2, 1, 1, 14, [3], None, 0, "half", dtype, 32, 42, tweak)


def attention_case(D, n_q, n_kv, B, n, base, lens, page, seed, scale=None, pad=0, poison=False, max_ctx=None, hole=None,
                   loud=1.0):
    """One attention call on random rows, checked at every row against 64 bits."""
    top = max(b + (n if lens is None else l) for b, l in zip(base, [n] * B if lens is None else lens))
    max_ctx = max_ctx or top + 2
    slots = np.random.default_rng(seed).permutation(B + 1)[:B]
    cache = make_cache(2, n_kv, D, B + 1, max_ctx, page, seed)
    g = torch.Generator().manual_seed(seed + 1)
    all_slots = i32(slots)
    k = torch.randn((B, top, n_kv, D), generator=g).cuda() * loud
    v = torch.randn((B, top, n_kv, D), generator=g).cuda()
    sdrl.kv4_append(cache, 1, all_slots, k, v, lens=i32([b + (n if lens is None else l) for b, l in
                                                       zip(base, [n] * B if lens is None else lens)]))
    cache.check()
    kv_len = np.full(B + 1, 3, np.int32)
    kv_len[slots] = base
    cache.kv_len.copy_(i32(kv_len))
    if poison:                                                       # NaN groups wherever no row may look
        for b in range(B):
            hi = base[b] + (n if lens is None else lens[b])
            for p in range(hi, -(-max_ctx // page) * page):
                pg, t, r = int(cache.block_table[slots[b], p // page]), p % page // 32, p % 32
                cache.pages.view(torch.int32)[pg, 1, :, t, [8 * D + r, 8 * D + 32 + r]] = 0x7fc07fc0
    hc = host(cache)
    if hole is not None:
        cache.block_table[int(slots[hole[0]]), hole[1]] = -1
    q = torch.randn((B, n, n_q + pad, D), generator=g).bfloat16().cuda()[:, :, :n_q]
    out = torch.full((B, n, n_q + pad, D), 9.0, dtype=torch.bfloat16, device="cuda")
    ll = None if lens is None else i32(lens)
    sdrl.kv4_attention(cache, 1, all_slots, q, out[:, :, :n_q], scale=scale, lens=ll)
    got = out.float().cpu().numpy().astype(np.float64)
    qh = q.float().cpu().numpy().astype(np.float64)
    G, sc, worst = n_q // n_kv, D ** -0.5 if scale is None else scale, 0.0
    for b in range(B):
        m = n if lens is None else lens[b]
        assert (got[b, m:] == 9.0).all() and (got[b, :, n_q:] == 9.0).all()
        P = base[b] + m
        for h in range(n_kv if m else 0):
            kk, vv = (hc.rows(int(slots[b]), 1, h, min(P, max_ctx), is_v) for is_v in (False, True))
            keep = np.ones(min(P, max_ctx), bool)
            if hole is not None and hole[0] == b:
                keep[hole[1] * page:(hole[1] + 1) * page] = False
            for i in range(m):
                if base[b] + i >= max_ctx:
                    assert (got[b, i, h * G:(h + 1) * G] == 0).all()
                    continue
                kp = keep[:base[b] + i + 1]
                sel = [tuple(x[:base[b] + i + 1][kp] for x in t) for t in (kk, vv)]
                for gq in range(h * G, (h + 1) * G):
                    if not kp.any():
                        assert (got[b, i, gq] == 0).all()
                        continue
                    want, tol = ref.attend(qh[b, i, gq], sel[0], sel[1], int(kp.sum()), sc)
                    err, tol = np.abs(got[b, i, gq] - want), tol + 2.0 ** -8 * np.abs(want)
                    worst = max(worst, float((err / tol).max()))
                    assert (err <= tol).all(), (b, i, gq, float((err / tol).max()))
    say("attention", D, n_q, n_kv, B, n, "worst error / bound", round(worst, 3))
    return cache


HEADS = [(128, 32, 8), (128, 40, 8), (64, 4, 4), (64, 6, 2), (128, 16, 1)]


@pytest.mark.parametrize("D,n_q,n_kv", HEADS)
@pytest.mark.parametrize("n", [1, 5])
def test_attention_decode(D, n_q, n_kv, n):
    attention_case(D, n_q, n_kv, 3, n, [0, 31, 70], None, 32, 51)
    attention_case(D, n_q, n_kv, 2, n, [300, 127], [n, n // 2], 64, 52, pad=1, poison=True)


@pytest.mark.parametrize("base", [0, 1, 30, 31, 32, 33, 127, 128, 129, 255, 256, 700])
def test_attention_lengths(base):
    attention_case(128, 4, 2, 1, 1, [base], None, 64, 60 + base, poison=True)
    attention_case(64, 2, 2, 1, 3, [base], None, 32, 61 + base, poison=True)


@pytest.mark.parametrize("n", [2, 9, 16, 17, 33, 48, 49, 65])
def test_attention_query_tiles(n):
    """Every number of query tiles, slices with rows of one head and of several."""
    attention_case(128, 2, 1, 2, n, [40, 3], None, 32, 70 + n)
    attention_case(64, 3, 1, 2, n, [129, 0], [n, n - 1], 64, 71 + n, poison=True)


def test_attention_prefill():
    attention_case(128, 4, 2, 2, 150, [0, 77], [150, 101], 64, 81, poison=True)


def test_attention_batch_past_the_item_target():
    """More sequences than work-groups are wanted: whole sequences, one of them without rows."""
    base = [(37 * b) % 90 for b in range(150)]
    lens = [(b * 7) % 3 for b in range(150)]
    attention_case(64, 8, 8, 150, 2, base, lens, 32, 83)


def test_attention_of_many_sequences_cut_into_items():
    """One KV head, so fewer sequences than work-groups are wanted; more than 64 of them, lengths far apart."""
    base = [(211 * b) % 1500 if b % 9 else 0 for b in range(100)]
    lens = [(b * 5) % 4 for b in range(100)]
    attention_case(64, 4, 1, 100, 3, base, lens, 64, 101, poison=True)
    attention_case(128, 2, 1, 70, 1, base[:70], None, 32, 102)


@pytest.mark.parametrize("n", [15, 60])
def test_attention_of_many_rows_over_a_long_context(n):
    """Two slices of tiles, and rows divided among the waves, each with a context cut into several items."""
    attention_case(128, 4, 1, 2, n, [2500, 900], [n, n - 4], 64, 103 + n, poison=True)
    attention_case(64, 4, 1, 3, n, [0, 1333, 31], None, 32, 104 + n)


def test_attention_of_many_rows_that_fill_the_device():
    """Rows divided among the waves in two tiles each, the sequences as they come and longest first."""
    attention_case(128, 8, 4, 64, 65, [(13 * b) % 40 for b in range(64)], None, 32, 107)
    attention_case(64, 16, 4, 130, 17, [(37 * b) % 90 for b in range(130)], [17 - b % 18 for b in range(130)], 32, 108, poison=True)


def test_attention_scale_and_loud_keys():
    attention_case(128, 4, 1, 1, 4, [200], None, 64, 85, scale=0.25, loud=6.0)
    attention_case(64, 4, 2, 1, 4, [200], None, 64, 86, scale=-0.5)
    attention_case(64, 4, 2, 1, 2, [90], None, 64, 87, scale=0.0)


def test_attention_missing_page_is_masked_and_reported():
    for D, hole, base in ((128, 1, 150), (64, 0, 20)):
        cache = attention_case(D, 4, 2, 2, 2, [base, 60], None, 64, 91, hole=(0, hole))
        with pytest.raises(sdrl.SDError, match="block-table"):
            cache.check()
        cache.check()                                                # the report cleared it


def test_attention_rows_past_max_ctx():
    cache = attention_case(128, 4, 2, 2, 6, [58, 10], None, 32, 95, max_ctx=64)


def test_nan_keys_and_values_reach_the_rows_that_see_them():
    say("nan rows")
    cache = make_cache(1, 1, 128, 1, 64, 32, 3)
    k, v = torch.randn((1, 40, 1, 128)).cuda(), torch.randn((1, 40, 1, 128)).cuda()
    k[0, 38, 0, 7] = float("nan")
    v[0, 39, 0, 9] = float("inf")
    sdrl.kv4_append(cache, 0, i32([0]), k, v)
    cache.kv_len.fill_(36)
    q = torch.randn((1, 4, 2, 128)).bfloat16().cuda()
    out = sdrl.kv4_attention(cache, 0, i32([0]), q).float().cpu()
    assert torch.isfinite(out[0, :2]).all() and torch.isnan(out[0, 2:]).all()
    cache.kv_len.fill_(35)                                           # rows 36..38 of them: the NaN value is past all
    out = sdrl.kv4_attention(cache, 0, i32([0]), q).float().cpu()
    assert torch.isfinite(out[0, :3]).all() and torch.isnan(out[0, 3]).all()
    cache.check()


def test_device_range_errors():
    say("range errors")
    cache = make_cache(1, 2, 64, 3, 64, 32, 5)
    hc = host(cache)
    k = torch.randn((2, 4, 2, 64)).cuda()
    q = torch.randn((2, 4, 2, 64)).cuda()
    q_out = torch.full((2, 4, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    out, ko, vo = (torch.full_like(q_out, 9.0) for _ in range(3))

    def expect(match, slots, lens=None, start=None):
        for call in (lambda: sdrl.kv4_append(cache, 0, i32(slots), k, k, q, q_out, lens=lens),
                     lambda: sdrl.kv4_attention(cache, 0, i32(slots), q_out, out, lens=lens),
                     lambda: sdrl.kv4_read(cache, 0, i32(slots), start if start is not None else i32([0, 0]), ko, vo, lens=lens)):
            call()
            with pytest.raises(sdrl.SDError, match=match):
                cache.check()

    zero = i32([0, 0])
    # nothing may be written: the pool is compared at the end
    expect("slot index", [-1, 3], start=zero)
    assert bool((q_out == 0).all() and (out == 0).all() and (ko == 0).all() and (vo == 0).all())
    cache.kv_len.fill_(64)
    expect("position outside", [0, 1], start=i32([64, -9]))
    assert bool((q_out == 0).all() and (out == 0).all() and (ko == 0).all() and (vo == 0).all())
    cache.kv_len.fill_(-(1 << 31))
    expect("position outside", [0, 1], start=i32([-(1 << 31), (1 << 31) - 1]))
    cache.kv_len.fill_((1 << 31) - 1)
    expect("position outside", [0, 1], start=i32([(1 << 31) - 1, -5]))
    cache.kv_len.fill_(0)
    cache.block_table.fill_(cache.pages.shape[0])
    expect("block-table", [0, 1], start=zero)
    assert bool((out == 0).all() and (ko == 0).all() and (vo == 0).all())
    cache.block_table.fill_(-1)
    expect("row count", [0, 1], lens=i32([5, 1]), start=zero)
    expect("row count", [0, 1], lens=i32([-1, 0]), start=zero)
    same_pool(cache, hc)
    cache.block_table.copy_(torch.arange(6, dtype=torch.int32).reshape(3, 2))
    table = sdrl.rope_table(sdrl.RopeConfig(1e4, 64), 2)               # a table that ends before the rows
    sdrl.kv4_append(cache, 0, i32([0, 1]), k, k, q, q_out, rope=table)
    with pytest.raises(sdrl.SDError, match="rotary table"):
        cache.check()
    assert bool((q_out[:, 2:] == 0).all() and (q_out[:, :2] != 0).any())


@pytest.mark.parametrize("B", [2, 70])
@pytest.mark.parametrize("n", [1, 4, 80])
def test_lengths_out_of_range_end_at_once(B, n):
    """Whatever kv_len holds: rows without a place are zeros, and no kernel walks 2^31 positions for them."""
    say("lengths", B, n)
    cache = make_cache(1, 1, 64, B, 128, 32, 8)
    slots, q = i32(range(B)), torch.randn((B, n, 2, 64)).bfloat16().cuda()
    k, q_out, out = torch.randn((B, n, 1, 64)).bfloat16().cuda(), torch.empty_like(q), torch.empty_like(q)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for length in (-(1 << 31), -(1 << 31) + 100, -(1 << 24), -n, 128, 1 << 24, (1 << 31) - 100, (1 << 31) - 1):
        cache.kv_len.fill_(length)
        q_out.fill_(9.0), out.fill_(9.0)
        start.record()
        sdrl.kv4_append(cache, 0, slots, k, k, q, q_out)
        sdrl.kv4_attention(cache, 0, slots, q, out)
        end.record()
        with pytest.raises(sdrl.SDError, match="position outside"):
            cache.check()
        assert bool((out == 0).all() and (q_out == 0).all()) and start.elapsed_time(end) < 100
    if n < 4:
        return
    cache.kv_len.fill_(-2)                                           # rows from the third on are positions 0, 1, ..
    sdrl.kv4_append(cache, 0, slots, k, k, q, q_out)
    sdrl.kv4_attention(cache, 0, slots, q, out)
    with pytest.raises(sdrl.SDError, match="position outside"):
        cache.check()
    assert bool((out[:, :2] == 0).all() and (q_out[:, :2] == 0).all() and (q_out[:, 2:] == q[:, 2:]).all())
    cache.kv_len.fill_(0)
    want = sdrl.kv4_attention(cache, 0, slots, q[:, 2:].contiguous()).float()
    assert float((out[:, 2:].float() - want).abs().max()) <= 2.0 ** -6 * float(want.abs().max())


def test_row_counts_of_many_sequences_are_checked():
    say("row counts")
    cache = make_cache(1, 1, 64, 80, 64, 32, 6)
    slots, q = i32(range(80)), torch.zeros((80, 2, 2, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (-1, 3):
        lens = torch.full((80,), 2, dtype=torch.int32, device="cuda")
        lens[77] = bad
        sdrl.kv4_attention(cache, 0, slots, q, lens=lens)
        with pytest.raises(sdrl.SDError, match="row count"):
            cache.check()


def test_tensors_are_checked():
    """What the entry points refuse before a launch."""
    say("refusals")
    cache = make_cache(2, 2, 64, 3, 64, 32, 7)
    slots, lens = i32([0, 2]), i32([1, 3])
    bf = dict(dtype=torch.bfloat16, device="cuda")
    k, q, o = torch.zeros((2, 3, 2, 64), **bf), torch.zeros((2, 3, 4, 64), **bf), torch.zeros((2, 3, 4, 64), **bf)
    table = sdrl.rope_table(sdrl.RopeConfig(1e4, 64), 64)
    ws = torch.zeros(sdrl.kv4_workspace_bytes(cache, 2, 3, 4), dtype=torch.uint8, device="cuda")
    hc = host(cache)
    wide = torch.zeros((2, 3, 2, 72), **bf)[..., :64]                  # heads that are not contiguous
    skew = torch.zeros((2, 4, 2, 64), **bf)[:, :3]                     # sequences at another stride than n rows
    odd = torch.zeros(2 * 3 * 132, **bf).as_strided((2, 3, 2, 64), (396, 132, 64, 1))   # rows of 264 bytes
    app = dict(layer=0, slots=slots, k=k, v=k, q=q, q_out=o, rope=table, lens=lens)
    for kw in (dict(layer=2), dict(layer=-1), dict(slots=slots.long()), dict(slots=slots.cpu()), dict(slots=slots[:1]),
               dict(lens=i32([1])), dict(lens=lens.float()), dict(k=k.half()), dict(k=k.float()), dict(v=k.float()), dict(k=wide),
               dict(v=skew), dict(k=odd), dict(k=k[:, :2]), dict(k=k.cpu()), dict(q=None), dict(q_out=None), dict(q_out=o.float()),
               dict(q=q.float()), dict(q_out=o[:, :, :2]), dict(rope=table[..., :1]), dict(rope=table.double()),
               dict(rope=table[:, ::2]), dict(layout="pairs"), dict(k=k[..., :32], v=k[..., :32])):
        with pytest.raises((ValueError, sdrl.SDError)):
            sdrl.kv4_append(cache, **{**app, **kw})
    att = dict(layer=0, slots=slots, q=q, out=o, lens=lens, workspace=ws)
    for kw in (dict(layer=2), dict(slots=slots[:1]), dict(q=q.float()), dict(q=q[:, :, :3]), dict(out=o.float()),
               dict(out=o[:, :2]), dict(workspace=ws[:-256]), dict(workspace=ws[16:]), dict(workspace=ws.cpu()),
               dict(workspace=ws.float()), dict(scale=float("nan")), dict(lens=i32([1, 2, 3]))):
        with pytest.raises((ValueError, sdrl.SDError)):
            sdrl.kv4_attention(cache, **{**att, **kw})
    rd = dict(layer=0, slots=slots, start=slots, k_out=k, v_out=k.clone(), lens=lens)
    for kw in (dict(layer=2), dict(start=slots.long()), dict(start=slots[:1]), dict(k_out=k.float()), dict(v_out=k[:, :2]),
               dict(k_out=wide), dict(slots=slots.cpu())):
        with pytest.raises((ValueError, sdrl.SDError)):
            sdrl.kv4_read(cache, **{**rd, **kw})
    same_pool(cache, hc)
    cache.check()


def test_offsets_past_4_gb():
    """A pool of more than 2^32 bytes, its last page in use."""
    say("pool past 4 GB")
    D, n_kv, page = 128, 8, 128
    per_page = page * n_kv * 136
    n_pages = (1 << 32) // per_page + 40
    pages = sdrl.kv4_pages(n_pages, 1, n_kv, D, page)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2]], dtype=torch.int32, device="cuda")
    cache = sdrl.KV4Cache(pages, table, torch.zeros(1, dtype=torch.int32, device="cuda"), 3 * page)
    small = sdrl.KV4Cache(sdrl.kv4_pages(3, 1, n_kv, D, page), i32([[2, 0, 1]]), cache.kv_len, 3 * page)
    k, v = torch.randn((1, 300, n_kv, D)).cuda(), torch.randn((1, 300, n_kv, D)).cuda()
    q = torch.randn((1, 2, 32, D)).bfloat16().cuda()
    outs = []
    for c in (cache, small):
        c.kv_len.fill_(0)
        sdrl.kv4_append(c, 0, i32([0]), k, v)
        c.kv_len.fill_(298)
        outs.append(sdrl.kv4_attention(c, 0, i32([0]), q))
        c.check()
    assert torch.equal(outs[0], outs[1])
    assert torch.equal(pages[n_pages - 1], small.pages[2]) and torch.equal(pages[n_pages - 2], small.pages[1])


def _run_together(cache, slots, k, v, q, table, q_out, out, ws):
    sdrl.kv4_append(cache, 0, slots, k, v, q, q_out, rope=table)
    return sdrl.kv4_attention(cache, 0, slots, q_out, out, workspace=ws)


def test_together_on_a_stream_and_in_graphs():
    """Append and attention as a decode step runs them: on a side stream, and in two captured graphs with a workspace
    each, replayed in turn with eager work between, every replay against the eager result."""
    say("streams and graphs")
    D, n_q, n_kv, B = 128, 8, 2, 3
    cache = make_cache(1, n_kv, D, B, 700, 64, 7)
    table = sdrl.rope_table(sdrl.RopeConfig(5e5, D), 700)
    slots = i32(range(B))
    pk, pv = torch.randn((B, 600, n_kv, D)).cuda(), torch.randn((B, 600, n_kv, D)).cuda()
    sdrl.kv4_append(cache, 0, slots, pk, pv, rope=table)
    steps = []
    for n in (1, 4):
        x = torch.randn((B, n, n_q + 2 * n_kv, D)).bfloat16().cuda()
        steps.append(dict(q=x[:, :, :n_q], k=x[:, :, n_q:n_q + n_kv], v=x[:, :, n_q + n_kv:],
                          q_out=torch.empty((B, n, n_q, D), dtype=torch.bfloat16, device="cuda"),
                          out=torch.empty((B, n, n_q, D), dtype=torch.bfloat16, device="cuda"),
                          ws=torch.empty(sdrl.kv4_workspace_bytes(cache, B, n, n_q), dtype=torch.uint8, device="cuda")))

    def run(s):
        return _run_together(cache, slots, s["k"], s["v"], s["q"], table, s["q_out"], s["out"], s["ws"])

    lens = [i32([600, 411, 0]), i32([13, 600, 255])]
    before = cache.pages.clone()                       # a step writes rows that the next one's sequences may see
    want = []
    for ln in lens:
        cache.pages.copy_(before)
        cache.kv_len.copy_(ln)
        want.append([run(s).clone() for s in steps])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.pages.copy_(before)
        cache.kv_len.copy_(lens[0])
        on_side = [run(s).clone() for s in steps]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for a, b in zip(on_side, want[0]):
        assert torch.equal(a, b)
    graphs = []
    for s in steps:
        g = torch.cuda.CUDAGraph()
        with sdrl.no_collection(), torch.cuda.graph(g):
            run(s)
        graphs.append(g)
    for rep in range(4):
        ln = rep % 2
        cache.pages.copy_(before)
        cache.kv_len.copy_(lens[ln])
        for s, g, w in zip(steps, graphs, want[ln]):
            s["out"].zero_()
            g.replay()
            assert torch.equal(s["out"], w), rep
        torch.cuda.synchronize()
        (steps[0]["out"].float() + 1).sum().item()
    cache.check()


def test_two_calls_at_once():
    """Two attention calls on two streams, a workspace each, against the same calls one after the other."""
    say("two calls at once")
    cache = make_cache(1, 2, 128, 2, 3000, 64, 9)
    k, v = torch.randn((2, 2900, 2, 128)).cuda(), torch.randn((2, 2900, 2, 128)).cuda()
    sdrl.kv4_append(cache, 0, i32([0, 1]), k, v)
    cache.kv_len.copy_(i32([2890, 1777]))
    qs = [torch.randn((1, 5, 8, 128)).bfloat16().cuda() for _ in range(2)]
    want = [sdrl.kv4_attention(cache, 0, i32([b]), qs[b]).clone() for b in range(2)]
    slot = [i32([0]), i32([1])]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for b in range(2):
            with torch.cuda.stream(streams[b]):
                got[b].append(sdrl.kv4_attention(cache, 0, slot[b], qs[b]))
    torch.cuda.synchronize()
    for b in range(2):
        for o in got[b]:
            assert torch.equal(o, want[b])
