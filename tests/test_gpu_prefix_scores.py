"""The group attention at scores of any size: past 2^24 a unit in the last place of a score is no small part of the
softmax's range."""
import numpy as np
import pytest
import torch

from gpu_common import say
from prefix_ref import E24, HALF, Batch

pytestmark = pytest.mark.gpu


def set_keys(x, b, keys):
    """Sequence b's keys [positions][n_kv][D], in its pages too (the groups' first positions: of all of them alike)."""
    x.K[b] = keys.bfloat16().contiguous()
    P = np.arange(len(keys))
    pg = x.table[int(x.slots_h[b])].long()[torch.from_numpy(P // x.page).cuda()]
    x.k[pg, x.layer, :, torch.from_numpy(P % x.page).cuda()] = x.K[b]


def check(x, out, b):
    """Rows of sequence b against 64 bits; the number of them (of heads) without a statement, and of all.  A score is off by its
    sum of D products in fp32 and the product with scale log2 e, 2^-24 (D + 8) of the sum of their sizes.  Where that
    is below 2^-6, a weight is off by twice as much of itself.  Where it is more, but one position is ahead of all others
    by more than it and 25, that has all the weight: the others' e^-25 each is added to the bound."""
    G, m, D = x.n_q // x.n_kv, int(x.lens_h[b]), x.D
    q = x.q[b, :m].double()
    K, V = (t.double().repeat_interleave(G, 1) for t in (x.K[b], x.V[b]))
    s = torch.einsum("ihd,phd->hip", q, K) * D ** -0.5
    err = torch.einsum("ihd,phd->hip", q.abs(), K.abs()) * D ** -0.5 * E24 * (D + 8)
    pos = torch.arange(len(K), device=q.device)
    seen = (pos[None] <= int(x.base[b]) + torch.arange(m, device=q.device)[:, None])[None]
    s, err = torch.where(seen, s, -torch.inf), torch.where(seen, err, 0.0)
    weigh = (s + err) > (s - err).amax(-1, keepdim=True) - 25
    off = torch.where(weigh, err, 0.0).amax(-1)                                 # [n_q, m]
    fine, alone = off < 2.0 ** -6, weigh.sum(-1) == 1
    p = torch.softmax(s, -1)
    o, a = torch.einsum("hip,phd->ihd", p, V), torch.einsum("hip,phd->ihd", p, V.abs())
    off = torch.where(fine, off, 0.0).t()[..., None]
    tol = a * (HALF + 2 * off + E24 * (len(K) / 16 + 64)) + HALF * o.abs() * (1 + 2 * HALF) + len(K) * np.exp(-25.0) * V.abs().amax(0) + 1e-30
    said = (fine | alone).t()[..., None].expand_as(o)
    got = out[b, :m].double()
    assert bool(torch.isfinite(got).all()), b
    bad = ((got - o).abs() > tol) & said
    assert not bool(bad.any()), (b, bad.any(-1).nonzero()[:4].tolist(), float(((got - o).abs() / tol)[said].max()))
    return int((~(fine | alone)).sum()), fine.numel()


# heads, sequences, shared positions, rows: few and many rows of a slice, work-groups that walk several sequences, several
# slices of one sequence
FORMS = [(8, 2, 128, [4], 700, 2), (32, 8, 128, [8], 1000, 5), (64, 64, 64, [20], 1000, 1), (256, 32, 128, [7], 900, 3),
         (8, 2, 64, [3], 200, 70), (4, 4, 64, [1, 2], 130, 1)]


def form(n_q, n_kv, D, sizes, prefix, n, seed=0):
    own = np.random.default_rng(seed + 5).integers(0, 331, sum(sizes)).tolist()
    return Batch(n_q, n_kv, D, sizes, [prefix] * len(sizes), own, n, seed=seed)


@pytest.mark.parametrize("n_q,n_kv,D,sizes,prefix,n", FORMS)
@pytest.mark.parametrize("k", [10, 20, 24, 27, 31, 33, 40, 64, 100])
def test_large_queries(n_q, n_kv, D, sizes, prefix, n, k):
    x = form(n_q, n_kv, D, sizes, prefix, n)
    x.q *= 2.0 ** k
    for groups in (True, False):
        out, none, rows = x.run(groups=groups), 0, 0
        for b in range(0, x.B, 3):
            c = check(x, out, b)
            none, rows = none + c[0], rows + c[1]
        # (of 700 scores of 2^10 the two largest are nearer than 25 in 8 of 100 rows, of larger ones in fewer)
        assert none < 0.2 * rows, (none, rows)


@pytest.mark.parametrize("n_q,n_kv,D,sizes,prefix,n", FORMS)
def test_large_queries_beside_others(n_q, n_kv, D, sizes, prefix, n):
    """Rows of very different sizes in one wave."""
    x = form(n_q, n_kv, D, sizes, prefix, n, seed=1)
    for h, k in ((0, 40), (1, 0), (2, 26), (3, 64)):
        x.q[:, :, h::5] *= 2.0 ** k
    x.q[::2, :, 4::5] *= 2.0 ** 33
    out = x.run()
    none = sum(check(x, out, b)[0] for b in range(x.B))
    say("rows without a statement", none)


@pytest.mark.parametrize("n_q,n_kv,D,sizes,prefix,n", FORMS)
@pytest.mark.parametrize("k", [0, 31, 40, 90])
@pytest.mark.parametrize("sign", [1, -1])
def test_equal_scores_of_any_size(n_q, n_kv, D, sizes, prefix, n, k, sign):
    """One key at every position: the values' mean, whatever the scores' size and sign."""
    x = form(n_q, n_kv, D, sizes, prefix, n, seed=2)
    key = torch.randn((n_kv, D), generator=torch.Generator().manual_seed(3)).cuda()
    for b in range(x.B):
        set_keys(x, b, key.expand(len(x.K[b]), -1, -1))
    x.q.copy_(sign * (key.repeat_interleave(n_q // n_kv, 0) * 2.0 ** k).expand_as(x.q))
    out = x.run()
    for b in range(0, x.B, 3):
        V = x.V[b].double().repeat_interleave(n_q // n_kv, 1)
        for i in range(0, n, 7):
            m = int(x.base[b]) + i + 1
            o, a = V[:m].mean(0), V[:m].abs().mean(0)
            # one rounding of the one weight that all positions have, sums in fp32, the output's rounding
            tol = a * (HALF + E24 * (m / 16 + 64)) + HALF * o.abs() * (1 + 2 * HALF)
            assert bool(((out[b, i].double() - o).abs() <= tol).all()), (b, i)


@pytest.mark.parametrize("n_q,n_kv,D,sizes,prefix,n", FORMS)
@pytest.mark.parametrize("up", [True, False])
def test_scores_that_grow_or_shrink_on_the_way(n_q, n_kv, D, sizes, prefix, n, up):
    """Scores of ordinary size at one end of the cache and of 2^40 at the other: references that pass from one
    arithmetic to the other, and back for no row."""
    x = form(n_q, n_kv, D, sizes, prefix, n, seed=4)
    x.q *= 2.0 ** 40
    top = max(len(t) for t in x.K)
    for b in range(x.B):
        e = torch.arange(len(x.K[b]), device="cuda") / top * 40
        set_keys(x, b, x.K[b].float() * torch.exp2(e - 40 if up else -e)[:, None, None])
    out = x.run()
    for b in range(0, x.B, 3):
        check(x, out, b)
