"""Argument checks of the rotary tables and the 4-bit KV cache that need no GPU: every refusal of the C entries
comes before a launch, and the reference the GPU tests use agrees with itself."""
import ctypes as C

import numpy as np
import pytest
import torch

import kv4_ref as ref
from paper_2606_18967_amd import sdrl, synth

BUF = (C.c_char * 8192)()
PTR = (C.addressof(BUF) + 255) & ~255                  # never dereferenced: refused calls launch nothing
INVAL, UNSUPPORTED = sdrl.SD_E_INVAL, sdrl.SD_E_UNSUPPORTED


def cache(**kw):
    d = dict(pages=PTR, block_table=PTR, kv_len=PTR, flags=None, n_pages=8, page_size=64, pages_per_seq=4, n_layers=2,
             n_kv=2, head_dim=128, max_slots=4, max_ctx=256)
    d.update(kw)
    return sdrl.KV4Struct(*d.values())


def test_page_bytes():
    f = sdrl.lib().sd_kv4_page_bytes
    assert f(2, 8, 128, 64) == 2 * 8 * 64 * 136
    assert f(1, 1, 64, 32) == 32 * 72
    for bad in ((0, 1, 64, 32), (1, 0, 64, 32), (1, 1, 96, 32), (1, 1, 64, 0), (1, 1, 64, 48)):
        assert f(*bad) == 0


@pytest.mark.parametrize("kw", [dict(pages=None), dict(block_table=None), dict(kv_len=None), dict(pages=PTR + 8),
                                dict(n_pages=0), dict(page_size=48), dict(page_size=0), dict(pages_per_seq=3),
                                dict(pages_per_seq=0), dict(n_layers=0), dict(n_kv=0), dict(head_dim=96), dict(max_slots=0),
                                dict(max_ctx=0), dict(max_ctx=257), dict(max_ctx=(1 << 30) + 64, pages_per_seq=1 << 30)],
                         ids=str)
def test_cache_is_checked(kw):
    L, c = sdrl.lib(), cache(**kw)
    assert L.sd_kv4_append(C.byref(c), 0, 1, 1, PTR, None, 1, PTR, 256, PTR, 256, None, 0, 0, None, None, None) == INVAL
    assert L.sd_kv4_read(C.byref(c), 0, 1, 1, PTR, PTR, None, PTR, PTR, None) == INVAL
    assert L.sd_kv4_workspace_bytes(C.byref(c), 1, 1, 4) == 0
    assert L.sd_kv4_attention(C.byref(c), 0, 1, 1, PTR, None, 4, PTR, 512, 1.0, PTR, 512, PTR, 1 << 20, None) == INVAL
    assert L.sd_last_error()


def test_append_is_checked():
    L = sdrl.lib()

    def call(c=None, layer=0, B=1, n=1, slots=PTR, dtype=1, k=PTR, k_ld=256, v=PTR, v_ld=256, q=PTR, q_ld=512, n_q=4,
             q_out=PTR, rope=None):
        c = c or cache()
        return L.sd_kv4_append(C.byref(c), layer, B, n, slots, None, dtype, k, k_ld, v, v_ld, q, q_ld, n_q, q_out, rope, None)

    for kw in (dict(layer=-1), dict(layer=2), dict(B=0), dict(B=5), dict(n=0), dict(n=257), dict(slots=None), dict(dtype=2),
               dict(k=None), dict(v=None), dict(k=PTR + 2), dict(v=PTR + 4), dict(k_ld=248), dict(v_ld=255), dict(k_ld=260),
               dict(dtype=0, k_ld=258), dict(q=None), dict(q_out=None), dict(n_q=0), dict(q_ld=504), dict(q_ld=516),
               dict(q=PTR + 8), dict(q_out=PTR + 8), dict(k_ld=1 << 40)):
        assert call(**kw) == INVAL, kw
    for args in ((PTR, 64, 8, 0), (PTR, 64, 136, 0), (PTR, 64, -16, 0), (None, 64, 64, 0), (PTR + 8, 64, 64, 0), (PTR, 0, 64, 0)):
        assert call(rope=C.byref(sdrl.RopeArgs(*args))) == INVAL, args
    big = cache(max_slots=1 << 20, max_ctx=1 << 20, pages_per_seq=1 << 15)
    assert call(big, B=1 << 20, n=1 << 20) == UNSUPPORTED
    small = cache(max_slots=128, max_ctx=1 << 20, pages_per_seq=1 << 15, n_kv=1, head_dim=64)   # mostly query rows
    assert call(small, B=128, n=1 << 20, n_q=1) == UNSUPPORTED


def test_read_and_attention_are_checked():
    L, c = sdrl.lib(), cache()
    assert L.sd_kv4_read(None, 0, 1, 1, PTR, PTR, None, PTR, PTR, None) == INVAL
    for start, k, v in ((None, PTR, PTR), (PTR, None, PTR), (PTR, PTR, None), (PTR, PTR + 2, PTR)):
        assert L.sd_kv4_read(C.byref(c), 0, 1, 1, PTR, start, None, k, v, None) == INVAL
    need = L.sd_kv4_workspace_bytes(C.byref(c), 2, 3, 4)
    assert need > 0 and L.sd_kv4_workspace_bytes(C.byref(c), 2, 3, 3) == 0

    def call(layer=0, B=2, n=3, slots=PTR, n_q=4, q=PTR, q_ld=512, scale=1.0, out=PTR, out_ld=512, ws=PTR, nb=need):
        return L.sd_kv4_attention(C.byref(c), layer, B, n, slots, None, n_q, q, q_ld, scale, out, out_ld, ws, nb, None)

    for kw in (dict(layer=2), dict(B=0), dict(n=0), dict(slots=None), dict(n_q=3), dict(n_q=0), dict(q=None), dict(q=PTR + 8),
               dict(q_ld=508), dict(q_ld=504), dict(scale=float("nan")), dict(scale=float("inf")), dict(out=None),
               dict(out=PTR + 2), dict(out_ld=500), dict(ws=None), dict(ws=PTR + 16), dict(nb=need - 1)):
        assert call(**kw) == INVAL, kw
    big = cache(max_slots=1 << 20, max_ctx=1 << 20, pages_per_seq=1 << 15)
    assert L.sd_kv4_workspace_bytes(C.byref(big), 70000, 1, 4) == 0
    assert L.sd_kv4_attention(C.byref(big), 0, 70000, 1, PTR, None, 4, PTR, 512, 1.0, PTR, 512, PTR, 1 << 40, None) == UNSUPPORTED


def test_rope_is_checked():
    L = sdrl.lib()
    ok = dict(theta=1e4, factor=2.0, low=1.0, high=4.0, attn_factor=0.0, rot_dim=64, scaling=2, orig_ctx=2048, reserved=0)

    def call(n=4, table=PTR, **kw):
        c = sdrl.RopeCfg(*{**ok, **kw}.values())
        return L.sd_rope_table(C.byref(c), n, table, None)

    nan, inf = float("nan"), float("inf")
    for kw in (dict(theta=1.0), dict(theta=nan), dict(theta=inf), dict(factor=0.5), dict(factor=nan), dict(factor=inf),
               dict(low=0.0), dict(high=1.0), dict(high=inf), dict(low=nan), dict(attn_factor=-1.0), dict(attn_factor=0.5),
               dict(scaling=3, attn_factor=nan), dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=258), dict(scaling=4),
               dict(scaling=-1), dict(orig_ctx=0), dict(reserved=1), dict(n=0), dict(n=(1 << 30) + 1), dict(table=None),
               dict(table=PTR + 4)):
        assert call(**kw) == INVAL, kw
    assert L.sd_rope_table(None, 4, PTR, None) == INVAL
    assert L.sd_set_rope(None, None, None) == INVAL and L.sd_bind_kv4(None, None) == INVAL
    with pytest.raises(ValueError):
        sdrl.RopeConfig(1e4, 64, "ntk")


def test_python_cache_is_checked():
    pages = sdrl.kv4_pages(4, 1, 2, 64, 32, device="cpu")
    assert pages.shape == (4, 1, 2, 1, 2304)
    t, n = torch.zeros((2, 2), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for p, tb, kl, ctx in ((pages[0], t, n, 64), (pages[..., :2300], t, n, 64), (pages, t, n, 65), (pages, t[0], n, 64),
                           (pages, t, n, 64)):                     # the last: not on a device
        with pytest.raises(ValueError):
            sdrl.KV4Cache(p, tb, kl, ctx)
    with pytest.raises(ValueError):
        sdrl.kv4_pages(4, 1, 2, 64, 48, device="cpu")


def test_reference_packing():
    """The reference's tile holds what is put in, one position at a time, and words and bits are where the format says."""
    rng = np.random.default_rng(0)
    for D in (64, 128):
        t = np.zeros(ref.tile_words(D), np.uint32)
        want = {}
        for r in rng.permutation(32):
            for is_v in (False, True):
                c, s, z = ref.quantize(rng.normal(size=D).astype(np.float32))
                ref.put(t, int(r), is_v, c, s, z)
                want[int(r), is_v] = (c, s, z)
        for (r, is_v), (c, s, z) in want.items():
            got = ref.get(t, r, is_v, D)
            assert np.array_equal(got[0], c) and got[1] == s and got[2] == z
        c = want[9, False][0]
        assert (int(t[9 * (D // 8) + 1]) >> 20) & 15 == c[8 + 3]       # dim 11: element 3 of word 1, bit 4 + 16
        c = want[13, True][0]
        assert (int(t[4 * D + D + 17]) >> 24) & 15 == c[17]            # position 13: element 5 of group 1, bit 8 + 16


def test_reference_quantizer_error():
    """Half a step a value, and what rounding s and z to bf16 can move the ends by."""
    rng = np.random.default_rng(1)
    y = (rng.normal(size=(500, 128)) * np.exp(rng.normal(size=(500, 1)) * 3)).astype(np.float32)
    c, s, z = ref.quantize(y)
    back = z[:, None].astype(np.float64) + s[:, None].astype(np.float64) * (c - 8)
    tol = s.astype(np.float64) * (0.5 + 15 * 2.0 ** -8) + np.abs(z) * 2.0 ** -8
    assert (np.abs(back - y) <= tol[:, None]).all() and c.min() == 0 and c.max() == 15
