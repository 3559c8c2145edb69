"""Rows of the 4-bit attention that must not depend on their neighbours: rows past the cache's last position where a
sequence is cut into items, next to queries that are infinite, NaN or of far larger size; every row against 64 bits
under the bound of the kernel's own arithmetic."""
import numpy as np
import pytest
import torch

import kv4_ref as ref
from paper_2606_18967_amd import sdrl

from gpu_common import i32, say
from test_gpu_kv4 import attention_case, host, make_cache, same_pool

pytestmark = pytest.mark.gpu


def filled(D, n_kv, B, ctx, max_ctx, page, seed, loud=1.0):
    """A cache whose slots hold ctx random positions, and its values on the host by slot and KV head:
    (codes - 8 [ctx][D], s [ctx], z [ctx]) of K and V in float64."""
    cache = make_cache(1, n_kv, D, B, max_ctx, page, seed)
    g = torch.Generator().manual_seed(seed + 1)
    k, v = (torch.randn((B, ctx, n_kv, D), generator=g) for _ in range(2))
    sdrl.kv4_append(cache, 0, i32(range(B)), (k * loud).cuda(), v.cuda())
    cache.check()
    hc = host(cache)
    return cache, [[tuple(hc.rows(b, 0, h, ctx, is_v) for is_v in (False, True)) for h in range(n_kv)] for b in range(B)]


def attend(q, k, v, scale):
    """Attention of q [D] over k, v = (c, s, z) in 64 bits, the bound on what the kernel may be off, and None, or the
    position that takes all the weight, where no smaller bound on the scores is needed.  The kernel's roundings:
    - a score, in fp32: 16 half steps (2^-24) of its terms' sizes, and the factor scale log2 e rounded to fp32;
    - P s in fp16: 2^-11 of each, and 2^-28 of the largest for the ones below fp16's normal numbers;
    - sums over codes 0..15 and the centre's eight of them in fp32: a half step for each tile of 32 positions and 8 more;
    - P, its sum and the merges in fp32: 2^-18;   - the output in bf16: 2^-8."""
    (kc, ks, kz), (vc, vs, vz) = k, v
    sc = scale * (ks * (kc @ q) + kz * q.sum())
    size = abs(scale) * (ks * (15 * np.abs(q).sum() + 8 * abs(q.sum())) + np.abs(kz) * np.abs(q).sum())
    offs = 16 * 2.0 ** -24 * size + 2.0 ** -22 * np.abs(sc)
    weigh = np.flatnonzero(sc + offs > (sc - offs).max() - 25)     # the others weigh below e^-25 < 2^-36 whatever the roundings
    off = float(offs[weigh].max())
    p = np.exp(sc - sc.max())
    p /= p.sum()
    val = vs[:, None] * vc + vz[:, None]
    at = None
    if off > 2.0 ** -6:
        if len(weigh) > 1:                                         # one position, or no statement
            return None, None, None
        at, off = int(weigh[0]), 0.0
    ps = p * vs
    tiles = len(sc) / 32 + 8
    tol = (2.0 ** -11 * (ps @ np.abs(vc)) + 2.0 ** -28 * ps.max() * np.abs(vc).sum(0) + tiles * 2.0 ** -24 * 23 * ps.sum()
           + (2 * off + 2.0 ** -18) * (p @ np.abs(val)))
    want = p @ val
    return want, tol + 2.0 ** -8 * np.abs(want), at


def check_rows(got, q, vals, base, n_kv, max_ctx, scale, skip=()):
    """Every row of one sequence but those in skip (row, head); the number of rows without a statement."""
    n, n_q = q.shape[:2]
    G, none, worst = n_q // n_kv, 0, 0.0
    for i in range(n):
        for h in range(n_q):
            if (i, h) in skip:
                continue
            if base + i >= max_ctx:
                assert (got[i, h] == 0).all(), (i, h)
                continue
            k, v = (tuple(x[:base + i + 1] for x in t) for t in vals[h // G])
            want, tol, _ = attend(q[i, h], k, v, scale)
            if want is None:
                none += 1
                continue
            err = np.abs(got[i, h] - want)
            worst = max(worst, float((err / tol).max()))
            assert (err <= tol).all(), (i, h, float((err / tol).max()))
    say("worst error / bound", round(worst, 3))
    return none


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


# n_kv and n: one tile, two, two slices of two, rows divided among the waves; contexts cut into several items but for the last
@pytest.mark.parametrize("D,n_q,n_kv,n,max_ctx", [(128, 4, 1, 1, 2048), (128, 4, 1, 5, 2048), (64, 4, 2, 5, 1536),
                                                  (128, 8, 1, 5, 2048), (64, 2, 1, 80, 2048), (128, 4, 2, 4, 64)])
def test_rows_past_max_ctx_are_zeros(D, n_q, n_kv, n, max_ctx):
    say("past max_ctx", D, n_q, n_kv, n, max_ctx)
    cache, vals = filled(D, n_kv, 2, max_ctx, max_ctx, 32, 7)
    q = torch.randn((2, n, n_q, D), generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    for length in (max_ctx - n // 2, max_ctx, max_ctx + 700, 2 ** 31 - 1):
        cache.kv_len.copy_(i32([length, 40]))
        out = torch.full_like(q, 9.0)
        sdrl.kv4_attention(cache, 0, i32([0, 1]), q, out)
        if length + n > max_ctx:
            with pytest.raises(sdrl.SDError, match="position outside"):
                cache.check()
        cache.check()
        for b, base in ((0, length), (1, 40)):
            assert check_rows(f64(out[b]), f64(q[b]), vals[b], base, n_kv, max_ctx, D ** -0.5) == 0


LOUD = [float("inf"), -float("inf"), float("nan"), 2.0 ** 27, -2.0 ** 40, 2.0 ** 100, 2.0 ** 121, 2.0 ** -9, 2.0 ** -30, 0.0]


@pytest.mark.parametrize("D,n_q,n_kv,B,n,base", [(128, 4, 1, 2, 1, 1500), (128, 8, 2, 2, 5, 90), (64, 4, 4, 2, 5, 1300),
                                                 (128, 12, 1, 1, 4, 700), (64, 4, 2, 2, 50, 60), (128, 4, 1, 1, 70, 900)])
@pytest.mark.parametrize("other", LOUD)
def test_a_row_does_not_depend_on_its_neighbours(D, n_q, n_kv, B, n, base, other):
    """One row is not finite in one value, or of another size than the rest; the others are right all the same."""
    say("neighbours", D, n_q, n_kv, B, n, base, other)
    ctx = base + n
    cache, vals = filled(D, n_kv, B, ctx, ctx + 3, 32, 11)
    cache.kv_len.fill_(base)
    q = torch.randn((B, n, n_q, D), generator=torch.Generator().manual_seed(5))
    at = (n - 1, n_q - 1)                                          # the last position, which the others precede
    if np.isfinite(other):
        q[:, at[0], at[1]] *= other
    else:
        q[:, at[0], at[1], 3] = other
    q = q.bfloat16().cuda()
    got = f64(sdrl.kv4_attention(cache, 0, i32(range(B)), q))
    cache.check()
    for b in range(B):
        assert check_rows(got[b], f64(q[b]), vals[b], base, n_kv, ctx + 3, D ** -0.5, skip=[at]) == 0
        if not np.isfinite(other):
            assert np.isnan(got[b][at]).all()
        elif abs(other) <= 1.0:
            h = at[1] * n_kv // n_q
            want, tol, _ = attend(f64(q[b])[at], *vals[b][h], D ** -0.5)
            assert want is None or (np.abs(got[b][at] - want) <= tol).all()


def test_rows_of_every_size_side_by_side():
    """Rows from 2^-60 to 2^16 in one slice."""
    say("sizes side by side")
    D, n_q, n, base = 128, 4, 8, 600
    cache, vals = filled(D, 1, 1, base + n, base + n, 64, 13)
    cache.kv_len.fill_(base)
    q = torch.randn((1, n, n_q, D), generator=torch.Generator().manual_seed(6))
    q *= (2.0 ** torch.linspace(-60, 16, n * n_q)).reshape(1, n, n_q, 1)
    q = q.bfloat16().cuda()
    got = f64(sdrl.kv4_attention(cache, 0, i32([0]), q))[0]
    assert check_rows(got, f64(q[0]), vals[0], base, 1, base + n, D ** -0.5) == 0


@pytest.mark.parametrize("D,n_q,n_kv,n,base", [(128, 4, 1, 1, 1500), (64, 4, 2, 5, 700), (128, 8, 2, 6, 90), (64, 2, 1, 70, 900)])
@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 27, -2.0 ** 40, 2.0 ** 80, 2.0 ** 110])
def test_scores_of_every_size(D, n_q, n_kv, n, base, size):
    """Loud queries: one position takes all the weight and its value comes out, however large the scores are."""
    say("loud queries", D, n_q, n_kv, n, base, size)
    cache, vals = filled(D, n_kv, 1, base + n, base + n, 32, 17)
    cache.kv_len.fill_(base)
    q = (torch.randn((1, n, n_q, D), generator=torch.Generator().manual_seed(8)) * size).bfloat16().cuda()
    got = f64(sdrl.kv4_attention(cache, 0, i32([0]), q))[0]
    assert check_rows(got, f64(q[0]), vals[0], base, n_kv, base + n, D ** -0.5) <= n * n_q // 8 + 1   # ties within fp32's last places


def test_loud_keys_that_come_late():
    """Ordinary scores first, then keys of 2^30 times the size, in a tile that every row sees whole and in the last ones."""
    say("late loud keys")
    D, n_q, base, n = 128, 4, 1000, 4
    for late in (500, 1001):
        cache = make_cache(1, 1, D, 1, base + n, 32, 19)
        g = torch.Generator().manual_seed(20)
        k, v = (torch.randn((1, base + n, 1, D), generator=g) for _ in range(2))
        k[0, late:] *= 2.0 ** 30
        sdrl.kv4_append(cache, 0, i32([0]), k.cuda(), v.cuda())
        cache.kv_len.fill_(base)
        hc = host(cache)
        vals = [tuple(hc.rows(0, 0, 0, base + n, is_v) for is_v in (False, True))]
        q = torch.randn((1, n, n_q, D), generator=g).bfloat16().cuda()
        got = f64(sdrl.kv4_attention(cache, 0, i32([0]), q))[0]
        assert check_rows(got, f64(q[0]), vals, base, 1, base + n, D ** -0.5) <= 2


def test_one_position_of_any_score():
    """A row that sees one position returns its value, also where the score is below -1e30."""
    say("one position")
    D = 128
    cache, vals = filled(D, 1, 2, 1, 64, 32, 23)
    for size in (1.0, 2.0 ** 100, 2.0 ** 110):
        for sign in (1, -1):
            cache.kv_len.zero_()
            q = (torch.randn((2, 1, 4, D), generator=torch.Generator().manual_seed(9)) * size * sign).bfloat16().cuda()
            got = f64(sdrl.kv4_attention(cache, 0, i32([0, 1]), q))
            for b in range(2):
                assert check_rows(got[b], f64(q[b]), vals[b], 0, 1, 64, D ** -0.5) == 0


def test_rows_whose_own_page_is_missing():
    """Nothing of them is stored and they read back as zeros; their queries are rotated, and attend what is there."""
    say("own page missing")
    D, n_q, n_kv, n, base = 128, 4, 2, 3, 62                       # positions 62, 63 and, on the missing page, 64
    cache = make_cache(1, n_kv, D, 1, 128, 64, 29)
    g = torch.Generator().manual_seed(30)
    x = torch.randn((1, n, n_q + 2 * n_kv, D), generator=g).bfloat16().cuda()
    q, k, v = x[:, :, :n_q], x[:, :, n_q:n_q + n_kv], x[:, :, n_q + n_kv:]
    table = sdrl.rope_table(sdrl.RopeConfig(1e4, D), 128)
    start = cache.pages.clone()
    outs = []
    for missing in (False, True):
        cache.pages.copy_(start)
        cache.kv_len.fill_(base)
        if missing:
            cache.block_table[0, 1] = cache.pages.shape[0]
        q_out = torch.full((1, n, n_q, D), 9.0, dtype=torch.bfloat16, device="cuda")
        ko = torch.full((1, n, n_kv, D), 9.0, dtype=torch.bfloat16, device="cuda")
        vo = ko.clone()
        lens = None if missing else i32([2])                       # the same rows stored as with the page missing
        sdrl.kv4_append(cache, 0, i32([0]), k, v, q, q_out, rope=table)
        if not missing:
            cache.check()
            cache.pages.copy_(start)
            sdrl.kv4_append(cache, 0, i32([0]), k, v, rope=table, lens=lens)
            hc = host(cache)
            cache.check()
        else:
            same_pool(cache, hc)
            sdrl.kv4_read(cache, 0, i32([0]), i32([base]), ko, vo)
            assert bool((ko[:, 2] == 0).all() and (vo[:, 2] == 0).all() and (ko[:, :2] != 0).any())
            with pytest.raises(sdrl.SDError, match="block-table"):
                cache.check()
        outs.append(q_out)
    assert torch.equal(outs[0], outs[1])
    cache = attention_case(128, 4, 2, 2, 2, [150, 60], None, 64, 92, hole=(0, 2))
    with pytest.raises(sdrl.SDError, match="block-table"):
        cache.check()


@pytest.mark.parametrize("D,n_q,n_kv,n,base,page", [(128, 32, 8, 1, 333, 64), (128, 40, 8, 5, 200, 64), (64, 4, 4, 4, 2500, 32),
                                                    (128, 4, 1, 12, 3000, 128), (64, 8, 1, 7, 61, 32), (128, 4, 2, 130, 77, 96),
                                                    (64, 6, 2, 40, 1100, 64), (128, 16, 1, 1, 4000, 64)])
@pytest.mark.parametrize("values", ["alike", "small", "large", "mixed", "shifted"])
def test_rows_within_the_kernels_own_bound(D, n_q, n_kv, n, base, page, values):
    """All forms of the kernel under attend()'s bound, whose term for P s is fp16's 2^-11: values of one size, of 2^-40 and
    2^40 times it, of sizes from 2^-20 to 2^20 position by position, and of a mean far from zero."""
    say("own bound", D, n_q, n_kv, n, base, values)
    B, top = 2, base + n
    cache = make_cache(1, n_kv, D, B, top + 5, page, 31)
    g = torch.Generator().manual_seed(32)
    k, v = (torch.randn((B, top, n_kv, D), generator=g) for _ in range(2))
    if values == "mixed":
        v *= 2.0 ** (40 * torch.rand((B, top, n_kv, 1), generator=g) - 20)
    elif values == "shifted":
        v += 20
    else:
        v *= {"alike": 1.0, "small": 2.0 ** -40, "large": 2.0 ** 40}[values]
    sdrl.kv4_append(cache, 0, i32(range(B)), k.cuda(), v.cuda())
    hc = host(cache)
    lens = [n, (n + 1) // 2]
    cache.kv_len.copy_(i32([base, base // 3]))
    q = torch.randn((B, n, n_q, D), generator=g).bfloat16().cuda()
    out = torch.full_like(q, 9.0)
    sdrl.kv4_attention(cache, 0, i32(range(B)), q, out, lens=i32(lens))
    cache.check()
    for b, start in enumerate((base, base // 3)):
        vals = [tuple(hc.rows(b, 0, h, top, is_v) for is_v in (False, True)) for h in range(n_kv)]
        assert bool((out[b, lens[b]:] == 9.0).all())
        assert check_rows(f64(out[b, :lens[b]]), f64(q[b, :lens[b]]), vals, start, n_kv, top + 5, D ** -0.5) == 0
