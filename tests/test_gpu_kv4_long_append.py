"""Appends with so many rows that a wave takes several KV heads one after the other (the next one's loads under way
while one is quantized, the last wave of a group with fewer heads): every byte of the pool against the format."""
import numpy as np
import pytest
import torch

import kv4_ref as ref
from paper_2606_18967_amd import sdrl

from gpu_common import i32, say
from test_gpu_kv4 import host, make_cache, same_pool

pytestmark = pytest.mark.gpu


def put_rows(hc, slot, layer, pos, is_v, codes, s, z):
    """HostCache.put of rows [m][n_kv] at consecutive positions, in one go."""
    D, P = hc.D, hc.P
    page, tile, r = hc.table[slot, pos // P], pos % P // 32, pos % 32
    bits = lambda x: np.where(np.isnan(x), 0x7fc0, x.view(np.uint32) >> 16).astype(np.uint32)
    par = bits(s) | bits(z) << np.uint32(16)
    codes = codes.astype(np.uint32)
    for h in range(codes.shape[1]):
        if is_v:
            at = 4 * D + (r // 8 * D)[:, None] + np.arange(D)
            for e in range(8):                                     # positions of one place in their words have words of their own
                k = np.flatnonzero(r % 8 == e)
                w = hc.w[page[k, None], layer, h, tile[k, None], at[k]]
                sh = np.uint32(ref.shift(e))
                hc.w[page[k, None], layer, h, tile[k, None], at[k]] = w & ~(np.uint32(15) << sh) | codes[k, h] << sh
        else:
            word = sum(codes[:, h, e::8] << np.uint32(ref.shift(e)) for e in range(8))
            hc.w[page[:, None], layer, h, tile[:, None], (r * (D // 8))[:, None] + np.arange(D // 8)] = word
        hc.w[page, layer, h, tile, 8 * D + (32 if is_v else 0) + r] = par[:, h]


def test_put_rows_is_put():
    say("put_rows")
    rng = np.random.default_rng(1)
    cache = make_cache(2, 3, 64, 2, 200, 64, 1)
    a, b = host(cache), host(cache)
    pos = 37 + np.arange(90)
    for is_v in (False, True):
        c, s, z = ref.quantize(rng.normal(size=(90, 3, 64)).astype(np.float32))
        put_rows(a, 1, 1, pos, is_v, c, s, z)
        for i, p in enumerate(pos):
            for h in range(3):
                b.put(1, 1, h, int(p), is_v, c[i, h], s[i, h], z[i, h])
    assert np.array_equal(a.w, b.w)


# (sequences, rows): waves of a head each past twice KV4_APPEND_WAVES, so 2, 2, 3, 4 heads a wave
@pytest.mark.parametrize("D,n_q,n_kv,B,n,rot,layout,dtype", [
    (128, 6, 3, 24, 460, 128, "half", torch.bfloat16), (64, 5, 5, 16, 420, 32, "interleaved", torch.float32),
    (64, 6, 3, 40, 600, 64, "half", torch.float32), (128, 8, 8, 16, 700, 128, "half", torch.bfloat16)])
def test_append_with_several_heads_a_wave(D, n_q, n_kv, B, n, rot, layout, dtype):
    say("long append", D, n_q, n_kv, B, n, layout, dtype)
    rng = np.random.default_rng(n)
    base = rng.integers(0, 90, B)
    lens = np.where(rng.random(B) < 0.5, n, rng.integers(0, n + 1, B))
    max_ctx, slots = int(base.max()) + n, rng.permutation(B)
    cache = make_cache(2, n_kv, D, B, max_ctx, 64, 3)
    kv_len = np.zeros(B, np.int32)
    kv_len[slots] = base
    cache.kv_len.copy_(i32(kv_len))
    hc = host(cache)
    x = torch.randn((B, n, n_q + 2 * n_kv, D), generator=torch.Generator().manual_seed(4)).to(dtype).cuda()
    q, k, v = x[:, :, :n_q], x[:, :, n_q:n_q + n_kv], x[:, :, n_q + n_kv:]
    table = sdrl.rope_table(sdrl.RopeConfig(1e4, rot), max_ctx)
    q_out = torch.full((B, n, n_q, D), 9.0, dtype=torch.bfloat16, device="cuda")
    sdrl.kv4_append(cache, 1, i32(slots), k, v, q, q_out, rope=table, layout=layout, lens=i32(lens))
    cache.check()
    tab, xh, qh = table.cpu().numpy(), x.float().cpu().numpy(), q_out.float().cpu().numpy()
    for b in range(B):
        m = int(lens[b])
        pos = base[b] + np.arange(m)
        yk = ref.rotate(xh[b, :m, n_q:n_q + n_kv], tab, pos[:, None], rot, layout)
        for is_v, y in ((False, yk), (True, xh[b, :m, n_q + n_kv:])):
            put_rows(hc, int(slots[b]), 1, pos, is_v, *ref.quantize(y))
        xq = xh[b, :m, :n_q]
        yq = ref.rotate(xq, tab, pos[:, None], rot, layout)
        # fp32 rotation (three roundings of up to |x| sqrt(2)), then bf16
        assert (np.abs(qh[b, :m] - yq) <= 2.0 ** -8 * np.abs(yq) + 2.0 ** -21 * np.abs(xq).max(initial=0.0)).all()
        assert (qh[b, m:] == 9.0).all()
    same_pool(cache, hc)
