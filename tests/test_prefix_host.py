"""Refusals of the calls over a paged bf16 cache and its groups, before anything is launched.  No GPU."""
import ctypes as C

import pytest
import torch

from paper_2606_18967_amd import sdrl

BUF = (C.c_char * 8192)()
PTR = (C.addressof(BUF) + 255) & ~255                  # never dereferenced: refused calls launch nothing
INVAL, UNSUPPORTED = sdrl.SD_E_INVAL, sdrl.SD_E_UNSUPPORTED


def cache(**kw):
    d = dict(k_pages=PTR, v_pages=PTR, block_table=PTR, kv_len=PTR, flags=None, n_pages=8, page_size=64, pages_per_seq=4, n_layers=2,
             n_kv=2, head_dim=128, max_slots=4, max_ctx=256)
    d.update(kw)
    return sdrl.KVStruct(*d.values())


@pytest.mark.parametrize("kw", [dict(k_pages=None), dict(v_pages=None), dict(block_table=None), dict(kv_len=None), dict(k_pages=PTR + 8),
                                dict(v_pages=PTR + 2), dict(n_pages=0), dict(page_size=48), dict(page_size=0), dict(pages_per_seq=3),
                                dict(n_layers=0), dict(n_kv=0), dict(head_dim=96), dict(max_slots=0), dict(max_ctx=0), dict(max_ctx=257),
                                dict(max_ctx=(1 << 24) + 1, pages_per_seq=1 << 30)], ids=str)
def test_cache_is_checked(kw):
    L, c = sdrl.lib(), cache(**kw)
    assert L.sd_kv_append(C.byref(c), 0, 1, 1, PTR, None, 1, PTR, 256, PTR, 256, None, 0, 0, None, None, None) == INVAL
    assert L.sd_prefix_workspace_bytes(C.byref(c), 1, 1, 4) == 0
    assert L.sd_prefix_attention(C.byref(c), None, 0, 1, 1, PTR, None, 4, PTR, 512, 1.0, PTR, 512, PTR, 1 << 30, None) == INVAL
    assert L.sd_last_error()


def test_append_is_checked():
    L = sdrl.lib()

    def call(c=None, layer=0, B=1, n=1, slots=PTR, dtype=1, k=PTR, k_ld=256, v=PTR, v_ld=256, q=PTR, q_ld=512, n_q=4, q_out=PTR, rope=None):
        c = c or cache()
        return L.sd_kv_append(C.byref(c), layer, B, n, slots, None, dtype, k, k_ld, v, v_ld, q, q_ld, n_q, q_out, rope, None)

    for kw in (dict(layer=-1), dict(layer=2), dict(B=0), dict(B=5), dict(n=0), dict(n=257), dict(slots=None), dict(dtype=2), dict(k=None),
               dict(v=None), dict(k=PTR + 2), dict(v=PTR + 4), dict(k_ld=248), dict(v_ld=255), dict(dtype=0, k_ld=258), dict(q=None),
               dict(q_out=None), dict(n_q=0), dict(q_ld=504), dict(q=PTR + 8), dict(q_out=PTR + 8), dict(k_ld=1 << 40)):
        assert call(**kw) == INVAL, kw
    for args in ((PTR, 64, 8, 0), (PTR, 64, 136, 0), (PTR, 64, -16, 0), (None, 64, 64, 0), (PTR + 8, 64, 64, 0), (PTR, 0, 64, 0)):
        assert call(rope=C.byref(sdrl.RopeArgs(*args))) == INVAL, args
    big = cache(max_slots=1 << 12, max_ctx=1 << 20, pages_per_seq=1 << 15)
    assert call(big, B=1 << 12, n=1 << 12) == UNSUPPORTED
    assert L.sd_kv_append(None, 0, 1, 1, PTR, None, 1, PTR, 256, PTR, 256, None, 0, 0, None, None, None) == INVAL


def test_attention_is_checked():
    L, c = sdrl.lib(), cache()
    need = L.sd_prefix_workspace_bytes(C.byref(c), 2, 3, 4)
    assert need > 0 and need % 256 == 0 and L.sd_prefix_workspace_bytes(C.byref(c), 2, 3, 3) == 0

    def call(layer=0, B=2, n=3, slots=PTR, n_q=4, q=PTR, q_ld=512, scale=1.0, out=PTR, out_ld=512, ws=PTR, nb=need, g=(PTR, PTR, 2, 0)):
        return L.sd_prefix_attention(C.byref(c), C.byref(sdrl.GroupsStruct(*g)), layer, B, n, slots, None, n_q, q, q_ld, scale, out,
                                     out_ld, ws, nb, None)

    for kw in (dict(layer=2), dict(layer=-1), dict(B=0), dict(B=5), dict(n=0), dict(slots=None), dict(n_q=3), dict(n_q=0), dict(q=None),
               dict(q=PTR + 8), dict(q_ld=508), dict(q_ld=504), dict(scale=float("nan")), dict(scale=float("inf")), dict(out=None),
               dict(out=PTR + 2), dict(out_ld=500), dict(ws=None), dict(ws=PTR + 16), dict(nb=need - 1), dict(g=(None, PTR, 2, 0)),
               dict(g=(PTR, None, 2, 0)), dict(g=(PTR, PTR, 0, 0)), dict(g=(PTR, PTR, 2, 1))):
        assert call(**kw) == INVAL, kw
    many = cache(max_slots=1 << 12)
    assert L.sd_prefix_workspace_bytes(C.byref(many), 1025, 1, 4) == 0
    assert L.sd_prefix_attention(C.byref(many), None, 0, 1025, 1, PTR, None, 4, PTR, 512, 1.0, PTR, 512, PTR, 1 << 40, None) == UNSUPPORTED


def test_calls_past_a_launch_are_refused():
    L, c = sdrl.lib(), cache(max_slots=64, max_ctx=1 << 21, pages_per_seq=1 << 15)
    # 2^20 rows of 8 heads a KV head are 2^16 slices; 7 x 2^20 x 16 rows of heads more than a launch has waves for
    for B, n, n_q in ((1, 1 << 20, 16), (7, 1 << 20, 16), (64, 1 << 19, 2)):
        assert L.sd_prefix_workspace_bytes(C.byref(c), B, n, n_q) == 0
        assert L.sd_prefix_attention(C.byref(c), None, 0, B, n, PTR, None, n_q, PTR, 128 * n_q, 1.0, PTR, 128 * n_q, PTR, 1 << 50,
                                     None) == UNSUPPORTED
    assert L.sd_prefix_workspace_bytes(C.byref(c), 1, 1 << 19, 16) > 0


def test_python_objects_are_checked():
    k = torch.zeros((4, 1, 2, 32, 64), dtype=torch.bfloat16)
    t, n = torch.zeros((2, 2), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for kk, tb, kl, ctx in ((k[0], t, n, 64), (k[..., :48], t, n, 64), (k[:, :, :, :31], t, n, 64), (k, t, n, 65), (k, t[0], n, 64), (k, t, n, 64)):
        with pytest.raises(ValueError):
            sdrl.KVPages(kk, kk, tb, kl, ctx)
    for g, ln in ((t, n), (n, t), (n, n[:0]), (n, n)):
        with pytest.raises(ValueError):
            sdrl.PrefixGroups(g, ln)


def test_a_workspace_serves_smaller_calls_too():
    L, c = sdrl.lib(), cache(max_slots=1024, max_ctx=4096, pages_per_seq=64, n_kv=8)
    f = lambda B, n: L.sd_prefix_workspace_bytes(C.byref(c), B, n, 32)  # noqa: E731
    for sizes in ([f(B, 5) for B in range(1, 1025)], [f(64, n) for n in range(1, 300)]):
        assert sizes[0] > 0 and sizes == sorted(sizes)
