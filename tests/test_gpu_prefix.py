"""Attention of groups that share a prompt, and the append, against 64 bits."""
import numpy as np
import pytest
import torch

import kv4_ref
from paper_2606_18967_amd import sdrl
from prefix_ref import E24, HALF, Batch

pytestmark = pytest.mark.gpu
HEADS = [(32, 8, 128), (40, 8, 128), (28, 4, 128), (16, 1, 128), (4, 2, 128), (4, 4, 64), (8, 2, 64)]


def own_lengths(sizes, top, seed):
    return np.random.default_rng(seed).integers(0, top + 1, sum(sizes)).tolist()


@pytest.mark.parametrize("n", [1, 2, 5])
@pytest.mark.parametrize("n_q,n_kv,D", HEADS)
def test_groups(n_q, n_kv, D, n):
    sizes = [3, 1, 8, 2]
    x = Batch(n_q, n_kv, D, sizes, [200, 130, 777, 64], own_lengths(sizes, 150, n), n, page=32 if n == 2 else 64)
    out = x.run()
    x.check(out)
    x.cache.check()
    alone = x.run(groups=False)
    x.check(alone)


@pytest.mark.parametrize("prefix", [0, 1, 31, 63, 64, 65, 127, 128, 191, 2048, 4097])
@pytest.mark.parametrize("page", [32, 96])
def test_prefix_lengths(prefix, page):
    x = Batch(8, 2, 64, [5], [prefix], [0, 1, 63, 64, 200], 1, page=page)
    x.check(x.run())


@pytest.mark.parametrize("sizes", [[1], [2], [1, 1, 1], [33], [64], [17, 40], [2] * 30])
@pytest.mark.parametrize("n", [1, 3])
def test_group_sizes(sizes, n):
    for prefix in (300, 800):
        x = Batch(8, 2, 128, sizes, [prefix] * len(sizes), own_lengths(sizes, 90, 1), n, seed=len(sizes))
        x.check(x.run())


@pytest.mark.parametrize("n_q,n_kv,D", [(32, 8, 128), (8, 2, 64)])
@pytest.mark.parametrize("n", [7, 70, 260])
def test_many_rows(n_q, n_kv, D, n):
    """Prefill-like blocks: several slices of rows, the causal limit inside each."""
    x = Batch(n_q, n_kv, D, [3, 2], [330, 64], [0, 3, 65, 0, 129], n, lens=[n, n // 2, 1, n - 1, n], seed=n)
    x.check(x.run())
    x.check(x.run(groups=False))


def test_ragged_rows_and_absent_sequences():
    sizes, n = [6, 4], 4
    x = Batch(28, 4, 128, sizes, [500, 129], own_lengths(sizes, 100, 3), n, lens=[4, 0, 1, 2, 0, 3, 0, 0, 4, 1])
    x.check(x.run())
    x.cache.check()


def test_only_absent_sequences():
    x = Batch(4, 2, 128, [2], [100], [3, 4], 2, lens=[0, 0])
    assert (x.run() == 7).all()


def test_batch_orders():
    """Members apart from one another, in any order: the same rows."""
    sizes = [4, 4]
    own = own_lengths(sizes, 80, 5)
    for order in ([0, 4, 1, 5, 2, 6, 3, 7], [7, 6, 5, 4, 3, 2, 1, 0], [0, 1, 4, 5, 6, 7, 2, 3]):
        x = Batch(8, 2, 128, sizes, [400, 333], own, 2, order=order)
        x.check(x.run())


def test_a_slot_twice():
    """Two blocks of rows of one sequence, side by side and apart."""
    for order in ([0, 1, 2, 3], [0, 2, 1, 3]):
        x = Batch(8, 2, 128, [4], [300], [10, 70, 130, 30], 2, order=order)
        a, b = order.index(0), order.index(1)
        x.slots[b] = x.slots[a]
        x.K[b], x.V[b], x.base[b] = x.K[a], x.V[a], x.base[a]
        x.check(x.run())
        x.cache.check()


def test_lengths_that_groups_do_not_have():
    """len past the shortest cache, 0 and negative; groups out of range."""
    sizes = [3, 3]
    own = [0, 100, 30, 10, 20, 30]
    x = Batch(8, 2, 128, sizes, [256, 200], own, 1)
    x.length.copy_(torch.tensor([1 << 30, -5], dtype=torch.int32))
    # of group 0 only 256 positions are alike: with len past that the contract is broken beyond the shortest kv_len,
    # which is 256 here
    x.check(x.run())
    x.length.zero_()
    x.check(x.run())
    x.group.fill_(99)
    x.check(x.run())
    x.group.fill_(-(1 << 31))
    x.check(x.run())


def test_many_sequences():
    sizes = [8] * 37 + [1, 7]
    x = Batch(4, 2, 128, sizes, [130] * len(sizes), own_lengths(sizes, 40, 2), 1)
    x.check(x.run(), seqs=[0, 1, 7, 8, 100, 295, 296, 303])
    assert not torch.isnan(x.run().float()).any()


@pytest.mark.parametrize("scale", [0.0, -0.1, 0.7])
def test_scales(scale):
    x = Batch(8, 2, 64, [4], [150], [3, 9, 70, 1], 2)
    x.check(x.run(scale=scale), scale=scale)


def test_strided_rows():
    x = Batch(8, 2, 64, [4], [150], [3, 9, 70, 1], 3)
    wide = torch.full((4, 3, 12, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((4, 3, 10, 64), dtype=torch.bfloat16, device="cuda")
    q[:, :, 1:9] = x.q
    out = wide[:, :, 2:10]
    x.run(q=q[:, :, 1:9], out=out)
    x.check(out)
    assert (wide[:, :, :2] == 7).all() and (wide[:, :, 10:] == 7).all()


def test_long_prefix():
    x = Batch(16, 1, 128, [6], [33000], [5, 100, 0, 700, 64, 1], 2)
    x.check(x.run(), seqs=[0, 3])
    x = Batch(28, 4, 128, [60], [9000], own_lengths([60], 300, 1), 1)
    x.check(x.run(), seqs=[0, 17, 59])


def test_peaked_scores():
    """Scores far apart: references move late in the walk, and most probabilities vanish."""
    x = Batch(8, 2, 128, [4], [700], [3, 9, 70, 1], 2)
    x.q *= 8
    x.check(x.run())


@pytest.mark.parametrize("n_q,n_kv,D,sizes,n", [(64, 64, 64, [20], 1), (64, 32, 128, [40], 2), (256, 32, 64, [20], 1), (64, 64, 128, [1, 1, 7], 3),
                                                (128, 128, 64, [70], 1)])
@pytest.mark.parametrize("peak", [1, 8])
@pytest.mark.parametrize("prefix", [200, 1000])
def test_chunks_over_several_sequences(n_q, n_kv, D, sizes, n, peak, prefix):
    """Many KV heads leave a head few work-groups: each walks the tiles of several sequences, whose rows have their first
    position and their references' moves at different tiles."""
    x = Batch(n_q, n_kv, D, sizes, [prefix] * len(sizes), own_lengths(sizes, 330, 5), n)
    x.q *= peak
    x.check(x.run(), seqs=range(0, sum(sizes), 3))


# few and many rows of a slice; behind short prompts sequences of many rows go alone
CHUNKS = [(64, 64, 64, 1, 0), (256, 32, 128, 3, 0), (256, 32, 128, 3, 12), (64, 64, 128, 12, 0), (64, 64, 128, 12, 12)]


@pytest.mark.parametrize("n_q,n_kv,D,n,more", CHUNKS)
@pytest.mark.parametrize("which,bad", [("k", float("nan")), ("k", float("inf")), ("v", float("nan")), ("v", -float("inf"))])
@pytest.mark.parametrize("tail", [70, 150])
def test_chunks_whose_values_are_not_finite(n_q, n_kv, D, n, more, which, bad, tail):
    """A key or value of sequence 1 behind its prompt, in a tile that all of its rows see or some: the others' are as before."""
    prefix = 200 + 64 * more
    x = Batch(n_q, n_kv, D, [7], [prefix], [170, tail, 0, 300, 64, 5, 130], n)
    x.q *= 4
    p, pool, G = prefix + 65, x.k if which == "k" else x.v, n_q // n_kv
    pool[int(x.table[int(x.slots_h[1]), p // x.page]), x.layer, 0, p % x.page, 5] = bad
    out = x.run()
    x.check(out, seqs=[0, 2, 3, 4, 5, 6])
    o, tol = x.expected(1)
    assert bool(((out[1].double() - o).abs() <= tol)[:, G:].all())
    if which == "v":
        assert not torch.isfinite(out[1, :, :G, 5]).any()
    elif bad != bad:
        assert torch.isnan(out[1, :, :G]).all()


@pytest.mark.parametrize("n_q,n_kv,D,n,more", CHUNKS)
def test_chunks_with_missing_pages(n_q, n_kv, D, n, more):
    x = Batch(n_q, n_kv, D, [7], [200 + 64 * more], [170, 150, 0, 300, 64, 5, 130], n)
    x.q *= 4
    for b, lp in ((0, 4 + more), (3, 7 + more), (6, 3 + more)):
        x.table[int(x.slots_h[b]), lp] = -1
        keep = torch.ones(len(x.K[b]), dtype=torch.bool, device="cuda")
        keep[64 * lp:64 * lp + 64] = False
        x.base[b] -= int((~keep)[:x.base[b] + 1].sum())            # (sequence 3's is its last page, rows and all)
        x.K[b], x.V[b] = x.K[b][keep], x.V[b][keep]
    x.check(x.run())


@pytest.mark.parametrize("n_q,n_kv,D,n,more", CHUNKS)
def test_chunks_with_ragged_rows(n_q, n_kv, D, n, more):
    x = Batch(n_q, n_kv, D, [5, 4], [200 + 64 * more, 90], [170, 150, 0, 300, 64, 5, 130, 61, 63], n, lens=[n, 0, 1, n, 0, n, 0, 1, n - 1])
    x.q *= 4
    x.check(x.run())


def test_scores_that_rise():
    """Keys that grow with the position, so that the reference moves in every tile."""
    x = Batch(4, 2, 64, [3], [640], [10, 20, 30], 1)
    x.q.copy_(x.q.abs())
    for b in range(3):
        ramp = (torch.arange(len(x.K[b]), device="cuda") / 40).bfloat16()[:, None, None].expand_as(x.K[b])
        x.K[b] = ramp.contiguous()
        P = np.arange(len(ramp))
        pg = x.table[int(x.slots_h[b])].long()[torch.from_numpy(P // x.page).cuda()]
        x.k[pg, x.layer, :, torch.from_numpy(P % x.page).cuda()] = x.K[b]
    x.check(x.run())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("which", ["k", "v"])
def test_what_is_not_finite_stays_with_the_rows_that_see_it(which, bad):
    """The last new row's key or value of sequence 1: its earlier rows do not see it."""
    n = 4
    x = Batch(8, 2, 128, [3], [300], [10, 20, 30], n)
    p = int(x.base[1]) + n - 1
    pool = x.k if which == "k" else x.v
    pool[int(x.table[int(x.slots_h[1]), p // x.page]), x.layer, 1, p % x.page, 5] = bad
    out = x.run()
    G = 4
    o, tol = x.expected(1)
    assert bool(((out[1, :n - 1].double() - o[:n - 1]).abs() <= tol[:n - 1]).all())
    assert bool(((out[1, n - 1, :G].double() - o[n - 1, :G]).abs() <= tol[n - 1, :G]).all())
    if which == "v" or bad != bad:
        assert torch.isnan(out[1, n - 1, G:]).all()
    x.B, keep = 1, x.B
    x.check(out)
    x.B = keep


def test_a_query_that_is_not_finite_stays_in_its_row():
    x = Batch(8, 2, 64, [3], [300], [10, 20, 30], 2)
    ref = x.run().clone()
    x.q[1, 0, 3, 7] = float("nan")
    x.q[2, 1, 5, 7] = float("inf")
    out = x.run()
    assert torch.isnan(out[1, 0, 3]).all() and torch.isnan(out[2, 1, 5]).all()
    out[1, 0, 3], out[2, 1, 5] = ref[1, 0, 3], ref[2, 1, 5]
    assert torch.equal(out, ref)


def test_bad_slots_positions_and_lengths_are_reported():
    n = 2
    x = Batch(8, 2, 64, [4], [100], [3, 9, 70, 1], n, max_ctx=192)
    ref = x.run().clone()
    x.cache.check()
    slots = x.slots.clone()
    x.slots[0] = 6
    out = x.run()
    with pytest.raises(sdrl.SDError, match="slot"):
        x.cache.check()
    assert (out[0] == 0).all()
    x.slots[0] = -1
    assert (x.run()[0] == 0).all()
    with pytest.raises(sdrl.SDError, match="slot"):
        x.cache.check()
    x.slots.copy_(slots)
    for length in (x.max_ctx - 1, x.max_ctx, (1 << 31) - 1, -1, -(1 << 31)):
        s = int(x.slots_h[3])
        keep = int(x.kv_len[s])
        x.kv_len[s] = length
        if length == x.max_ctx - 1:                    # its last position is there: a page of its own
            x.table[s, -1] = x.k.shape[0] - 1
            x.k[-1].zero_(), x.v[-1].zero_()
            x.table[s, x.table[s] < 0] = x.k.shape[0] - 1
        out = x.run()
        with pytest.raises(sdrl.SDError, match="position"):
            x.cache.check()
        assert (out[3, 1:] == 0).all() and (length == x.max_ctx - 1 or (out[3] == 0).all())
        assert all(bool(((out[b].double() - ref[b].double()).abs() <= 2 * x.expected(b)[1]).all()) for b in range(3))
        x.kv_len[s] = keep
    x.lens = torch.tensor([2, 3, -1, 2], dtype=torch.int32, device="cuda")
    x.lens_h = np.array([2, 2, 0, 2])
    x.check(x.run())
    with pytest.raises(sdrl.SDError, match="row count"):
        x.cache.check()


@pytest.mark.parametrize("where", ["shared", "own", "first"])
def test_missing_pages_are_as_if_masked(where):
    x = Batch(8, 2, 64, [3], [320], [10, 200, 30], 1, page=64)
    lp = dict(shared=2, own=6, first=0)[where]
    hit = [0, 1, 2] if where != "own" else [1]
    for b in hit:
        x.table[int(x.slots_h[b]), lp] = (-1, x.k.shape[0], 1 << 30)[b]
    out = x.run()
    with pytest.raises(sdrl.SDError, match="block-table"):
        x.cache.check()
    for b in hit:
        gone = slice(64 * lp, 64 * lp + 64)
        keep = torch.ones(len(x.K[b]), dtype=torch.bool, device="cuda")
        keep[gone] = False
        x.K[b], x.V[b] = x.K[b][keep], x.V[b][keep]
        x.base[b] -= 64
    x.check(out)


def test_no_page_at_all():
    x = Batch(8, 2, 64, [2], [128], [1, 2], 1)
    x.table.fill_(-1)
    assert (x.run() == 0).all()


def test_same_bits_again_and_in_parts():
    """Twice the same call, and each sequence's row with other sequences of its group beside it."""
    x = Batch(32, 8, 128, [8], [1000], own_lengths([8], 100, 0), 1)
    a, b = x.run(), x.run()
    assert torch.equal(a, b)


def test_in_a_graph_and_on_streams():
    x = Batch(32, 8, 128, [8, 4], [1000, 300], own_lengths([8, 4], 100, 0), 2)
    ws = [torch.empty(sdrl.prefix_workspace_bytes(x.cache, x.B, x.n, x.n_q), dtype=torch.uint8, device="cuda") for _ in range(2)]
    x.run(workspace=ws[0])
    side = torch.cuda.Stream()
    graphs, outs = [], [torch.zeros_like(x.q) for _ in range(2)]
    for k in range(2):
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with sdrl.no_collection(), torch.cuda.graph(graph, stream=side):
            x.run(workspace=ws[k], out=outs[k])
        torch.cuda.current_stream().wait_stream(side)
        graphs.append(graph)
    for seed in range(3):
        # other lengths of the cached positions and other shared ones: the plan is made on the device
        x.q.copy_(torch.randn(x.q.shape, device="cuda"))
        x.kv_len[x.slots.long()] = torch.from_numpy(x.base - seed).int().cuda()
        x.length.copy_(torch.tensor([1000 - 200 * seed, 300 - 64 * seed], dtype=torch.int32))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        eager = x.run()
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.current_stream())
            other = x.run()
        here = x.run()
        side.synchronize()
        for o in (*outs, other, here):
            assert torch.equal(o, eager)
        x.base -= seed
        x.K, x.V = [k[:len(k) - seed] for k in x.K], [v[:len(v) - seed] for v in x.V]
        x.check(eager)
        x.base += seed
        x.K, x.V = [torch.cat((k, torch.zeros_like(k[:seed]))) for k in x.K], [torch.cat((v, torch.zeros_like(v[:seed]))) for v in x.V]


def test_offsets_past_32_bits():
    """Pools of more than 2^32 bytes, the pages in use at their ends."""
    page_elems = 2 * 8 * 64 * 128
    n_pages = (1 << 32) // page_elems + 40                       # 2^32 elements and some
    if torch.cuda.mem_get_info()[0] < 5 * n_pages * page_elems * 2:
        pytest.skip("not enough memory")
    x = Batch(8, 8, 128, [4], [300], [10, 20, 30, 40], 1, pool_pages=n_pages)
    assert int(x.table.max()) * page_elems > 1 << 31
    x.check(x.run())


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n_q,n_kv,D,rot,layout,B,n,page", [(32, 8, 128, 128, "half", 8, 1, 64), (8, 2, 64, 32, "interleaved", 5, 33, 32),
                                                            (28, 4, 128, 0, "half", 3, 7, 96), (4, 4, 64, 64, "half", 1, 130, 32),
                                                            (16, 1, 128, 48, "interleaved", 4, 5, 64), (3, 1, 64, 16, "half", 2, 1, 32)])
def test_append(n_q, n_kv, D, rot, layout, B, n, page, dtype):
    rng = np.random.default_rng(B * n)
    base = rng.integers(0, 70, B)
    lens = np.concatenate(([n], rng.integers(0, n + 1, B - 1))) if n > 1 else None
    live = np.full(B, n) if lens is None else lens
    max_ctx = int(max(base) + n)
    per = -(-max_ctx // page)
    table = rng.permutation(B * per).reshape(B, per)
    k, v = (torch.full((B * per + 1, 2, n_kv, page, D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    i32 = lambda a: torch.from_numpy(np.asarray(a)).to(torch.int32).cuda()  # noqa: E731
    cache = sdrl.KVPages(k, v, i32(table), i32(base), max_ctx)
    rope = sdrl.rope_table(sdrl.RopeConfig(1e4, rot), max_ctx) if rot else None
    src = torch.randn((B, n, n_q + 2 * n_kv, D), generator=torch.Generator().manual_seed(n)).to(dtype).cuda()
    q_out = torch.full((B, n, n_q, D), 9.0, dtype=torch.bfloat16, device="cuda")
    sdrl.kv_append(cache, 1, i32(range(B)), src[:, :, n_q:n_q + n_kv], src[:, :, n_q + n_kv:], src[:, :, :n_q], q_out, rope=rope,
                   layout=layout, lens=None if lens is None else i32(lens))
    cache.check()
    want_k, want_v = k.clone(), v.clone()
    x = src.double().cpu().numpy()
    tab = rope.cpu().numpy() if rot else None
    for b in range(B):
        m = int(live[b])
        pos = base[b] + np.arange(m)
        turned = kv4_ref.rotate(x[b, :m, :n_q + n_kv], tab, np.repeat(pos[:, None], n_q + n_kv, 1), rot, layout) if m else np.zeros((0, n_q + n_kv, D))
        # two products and a sum in fp32, then bf16: half a step, and what the first may move over its border
        size = np.abs(x[b, :m, :n_q + n_kv]).max(-1, keepdims=True) * 2 if m else 0
        tol = HALF * np.abs(turned) * (1 + HALF) + 4 * E24 * size
        assert (np.abs(q_out[b, :m].double().cpu().numpy() - turned[:, :n_q]) <= tol[:, :n_q]).all()
        assert (q_out[b, m:] == 9).all()
        pg, at = torch.from_numpy(table[b, pos // page]).cuda(), torch.from_numpy(pos % page).cuda()
        got = k[pg, 1, :, at].double().cpu().numpy()
        assert (np.abs(got - turned[:, n_q:]) <= tol[:, n_q:]).all()
        assert torch.equal(v[pg, 1, :, at], src[b, :m, n_q + n_kv:].bfloat16())
        want_k[pg, 1, :, at], want_v[pg, 1, :, at] = k[pg, 1, :, at], v[pg, 1, :, at]
    assert torch.equal(k, want_k) and torch.equal(v, want_v)      # the others keep their contents


def test_append_reports_and_skips():
    k, v = (torch.full((4, 1, 1, 32, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.tensor([[0, 1], [2, -1], [3, 9]], dtype=torch.int32, device="cuda")
    cache = sdrl.KVPages(k, v, table, i32(63, 31, -1), 64)
    src = torch.ones((3, 2, 3, 64), dtype=torch.bfloat16, device="cuda")
    rope = sdrl.rope_table(sdrl.RopeConfig(1e4, 64), 64)
    call = lambda slots, **kw: sdrl.kv_append(cache, 0, slots, src[:, :, 1:2], src[:, :, 2:], src[:, :, :1], kw.pop("q_out", None), rope=rope, **kw)  # noqa: E731
    q = torch.full((3, 2, 1, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    call(i32(0, 1, 2), q_out=q)
    with pytest.raises(sdrl.SDError, match="position.*block-table|block-table.*position"):
        cache.check()
    assert (q[0, 1] == 0).all() and (q[2, 0] == 0).all()          # positions 64 and -1
    assert (v[1, 0, 0, 31] == 1).all() and (v[2, 0, 0, 31] == 1).all() and (v[3, 0, 0, 0] == 1).all()
    assert (v == 1).all(-1).sum() == 3 and (k != 9).any(-1).sum() == 3
    call(i32(-1, 3, 0), q_out=q)
    with pytest.raises(sdrl.SDError, match="slot"):
        cache.check()
    assert (q[:2] == 0).all()
    call(i32(0, 1, 2), q_out=q, lens=i32(3, -1, 0))
    with pytest.raises(sdrl.SDError, match="row count"):
        cache.check()


def test_append_without_queries_then_attend():
    """A decode step of two groups as a program runs it: append, then attend, against a call over the same cache
    filled by hand."""
    x = Batch(8, 2, 128, [3, 2], [200, 130], [5, 6, 70, 0, 9], 1)
    ref = x.run()
    rows = [torch.stack([kk[-1] for kk in src])[:, None] for src in (x.K, x.V)]
    for b in range(x.B):
        p = int(x.base[b])
        pg = int(x.table[int(x.slots_h[b]), p // x.page])
        x.k[pg, x.layer, :, p % x.page] = float("nan")
        x.v[pg, x.layer, :, p % x.page] = float("nan")
    sdrl.kv_append(x.cache, x.layer, x.slots, *rows)
    assert torch.equal(x.run(), ref)


def test_python_refusals():
    x = Batch(8, 2, 64, [2], [64], [1, 2], 1)
    bad = sdrl.PrefixGroups(x.group[:-1], x.length)
    with pytest.raises(ValueError):
        sdrl.prefix_attention(x.cache, bad, 1, x.slots, x.q)
    with pytest.raises(ValueError):
        x.run(q=x.q.float())
    with pytest.raises(ValueError):
        x.run(out=x.q.float())
    with pytest.raises(sdrl.SDError):
        x.run(workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(sdrl.SDError):
        sdrl.prefix_attention(x.cache, x.groups, 2, x.slots, x.q)
    with pytest.raises(ValueError):
        sdrl.PrefixGroups(x.group.long(), x.length)
