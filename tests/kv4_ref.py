"""The 4-bit cache's format and operators in plain numpy (64 bits), for its tests: packing of one tile at a time
as include/sd_api.h lays it out, rotation, quantization and attention by their formulas."""
import math

import numpy as np


def bf16(x):
    """Nearest bf16 value (ties to even) of float32 values, as float32."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7fff + ((u >> 16) & 1)) & 0xffff0000).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(x), np.float32(np.nan), r).astype(np.float32)


def frequencies(theta, rot, scaling="none", factor=1.0, low=0.0, high=0.0, orig=0, attn_factor=0.0):
    """Angle a position of each pair, and the factor of the table."""
    f, mul = [], 1.0
    for i in range(rot // 2):
        x = theta ** (-2.0 * i / rot)
        if scaling == "linear":
            x /= factor
        if scaling == "llama3":
            t = min(max((orig * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
            x *= t + (1 - t) / factor
        if scaling == "yarn":
            at = [rot * math.log(orig / (2 * math.pi * turns)) / (2 * math.log(theta)) for turns in (high, low)]
            a, b = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
            t = min(max((i - a) / max(b - a, 0.001), 0.0), 1.0)
            x *= (1 - t) + t / factor
            mul = attn_factor or 0.1 * math.log(factor) + 1.0
        f.append(x)
    return np.array(f), mul


def rotate(x, table, pos, rot, layout):
    """Rows x [..., D] float64 at positions pos [...] (table fp32 [p][rot/2][2]), rounded once to float32."""
    y = np.array(x, np.float64)
    if rot:
        i = np.arange(rot // 2)
        a, b = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
        c, s = (table[pos].astype(np.float64)[..., k] for k in (0, 1))
        xa, xb = np.array(x, np.float64)[..., a], np.array(x, np.float64)[..., b]
        y[..., a], y[..., b] = xa * c - xb * s, xa * s + xb * c
    return y.astype(np.float32)


def quantize(y):
    """Codes (int), s and z (float32) of rows y [..., D] float32; s = z = NaN where a row is not finite."""
    y = np.asarray(y, np.float32)
    ok = np.isfinite(y).all(-1)
    d = np.where(ok[..., None], y, 0).astype(np.float64)
    mn, mx = d.min(-1), d.max(-1)
    s = bf16(((mx - mn) / 15).astype(np.float32)).astype(np.float64)
    z = bf16((mn + 8 * s).astype(np.float32)).astype(np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.clip(np.rint((d - z[..., None]) / s[..., None]) + 8, 0, 15)
    c = np.where((s > 0)[..., None] & ok[..., None], c, 8).astype(np.int64)
    nan = np.float32(np.nan)
    return c, np.where(ok, s, nan).astype(np.float32), np.where(ok, z, nan).astype(np.float32)


def shift(e):
    return 4 * (e // 2) + 16 * (e % 2)


def tile_words(D):
    return 8 * (D + 8)


def put(tiles, r, is_v, codes, s, z):
    """Position r of a tile (uint32 words): codes [D], s, z."""
    D = len(codes)
    if is_v:
        at = 4 * D + r // 8 * D + np.arange(D)
        sh = shift(r % 8)
        tiles[at] = (tiles[at] & ~np.uint32(0xf << sh)) | (codes.astype(np.uint32) << np.uint32(sh))
    else:
        for w in range(D // 8):
            tiles[r * (D // 8) + w] = sum(int(codes[8 * w + e]) << shift(e) for e in range(8))
    bits = [0x7fc0 if np.isnan(x) else int(np.float32(x).view(np.uint32)) >> 16 for x in (s, z)]
    tiles[8 * D + (32 if is_v else 0) + r] = bits[0] | bits[1] << 16


def get(tiles, r, is_v, D):
    """(codes [D], s, z) of position r of a tile."""
    d = np.arange(D)
    if is_v:
        c = (tiles[4 * D + r // 8 * D + d] >> np.uint32(shift(r % 8))) & 15
    else:
        c = (tiles[r * (D // 8) + d // 8] >> shift(d % 8).astype(np.uint32)) & 15
    p = int(tiles[8 * D + (32 if is_v else 0) + r])
    s, z = (np.array([b << 16], np.uint32).view(np.float32)[0] for b in (p & 0xffff, p >> 16))
    return c.astype(np.int64), s, z


class HostCache:
    """The pages of a cache as uint32 words [n_pages][layers][n_kv][tiles][words]."""

    def __init__(self, pages, table, D):
        self.w = np.ascontiguousarray(pages).view(np.uint32).copy()
        self.table, self.D, self.P = table, D, 32 * pages.shape[3]

    def tile(self, slot, layer, h, p):
        return self.w[self.table[slot, p // self.P], layer, h, p % self.P // 32]

    def put(self, slot, layer, h, p, is_v, codes, s, z):
        put(self.tile(slot, layer, h, p), p % 32, is_v, codes, s, z)

    def get(self, slot, layer, h, p, is_v):
        return get(self.tile(slot, layer, h, p), p % 32, is_v, self.D)

    def rows(self, slot, layer, h, P, is_v):
        """codes - 8 [P][D], s [P], z [P] in float64 of the positions [0, P)."""
        got = [self.get(slot, layer, h, p, is_v) for p in range(P)]
        return (np.array([g[0] for g in got], np.float64).reshape(P, self.D) - 8, np.array([g[1] for g in got], np.float64),
                np.array([g[2] for g in got], np.float64))


def attend(q, k, v, see, scale):
    """Softmax attention of q [D] over positions [0, see) of k, v = (c, s, z), and the bound on what a kernel may be
    off that holds the probabilities times s in bf16 and the rest in 32 bits: the output's own rounding (2^-8) is the
    caller's; here 2^-8 of sum p s |c|, and 2^-14 of sum p |v| for scores and sums in fp32."""
    (kc, ks, kz), (vc, vs, vz) = [tuple(x[:see] for x in t) for t in (k, v)]
    sc = scale * (ks * (kc @ q) + kz * q.sum())
    p = np.exp(sc - sc.max())
    p /= p.sum()
    val = vs[:, None] * vc + vz[:, None]
    return p @ val, 2.0 ** -8 * (p @ np.abs(vs[:, None] * vc)) + 2.0 ** -14 * (p @ np.abs(val))


class Decoder:
    """One sequence through the decoder in 64 bits over a 4-bit cache, with the engine's roundings of what its
    kernels exchange: activations in bf16 (target) or fp16 (drafter), rotated queries in bf16, cached rows as their
    codes stand for.  weights: the binding order's tensors in float64; proj[l]: (Wqkv, Wo, Wgu, Wdown) to use."""

    def __init__(self, cfg, weights, proj, table, half=False):
        self.cfg, self.w, self.proj, self.table = cfg, weights, proj, table
        self.act = (lambda x: x.astype(np.float16).astype(np.float64)) if half else \
            (lambda x: bf16(x.astype(np.float32)).astype(np.float64))

    def norm(self, h, gain):
        return h / np.sqrt((h * h).mean(-1, keepdims=True) + self.cfg["rms_eps"]) * gain

    def forward(self, tokens, pos0, K, V, steps=None):
        """Logits [n][vocab] of tokens at pos0.., writing their rows into K, V [L][n_kv][cap][D] (values).  With the
        steps [L][n_kv][cap] of K and V given, their rows are there already, as the device stored them (one value near
        a border in another code is half a step, which would hide other errors): they must stand for the rows computed
        here to within half a step, s and z rounded to bf16, and 2e-2 of the row's largest value for the GEMM."""
        c = self.cfg
        nq, nkv, D, n = c["n_q"], c["n_kv"], c["head_dim"], len(tokens)
        pos = pos0 + np.arange(n)
        h = self.w[0][tokens]
        for l in range(c["n_layers"]):
            wqkv, wo, wgu, wdown = self.proj[l]
            x = (self.act(self.norm(h, self.w[3 + 6 * l])) @ wqkv.T).astype(np.float32).reshape(n, nq + 2 * nkv, D)
            q = bf16(rotate(x[:, :nq], self.table, pos[:, None], D, "half")).astype(np.float64)
            for buf, y in ((K, rotate(x[:, nq:nq + nkv], self.table, pos[:, None], D, "half")), (V, x[:, nq + nkv:])):
                if steps is not None:
                    s = steps[0 if buf is K else 1][l][:, pos]
                    got, y = buf[l][:, pos], y.swapaxes(0, 1).astype(np.float64)
                    top = np.abs(y).max(-1, keepdims=True)
                    assert (np.abs(got - y) <= 0.5 * s[..., None] + (2.0 ** -7 + 2e-2) * top).all(), (l, buf is K)
                    continue
                code, s, z = quantize(y)
                buf[l][:, pos] = (z[..., None].astype(np.float64) + s[..., None].astype(np.float64) * (code - 8)).swapaxes(0, 1)
            o = np.empty((n, nq, D))
            for i in range(n):
                for hh in range(nq):
                    kk, vv = K[l][hh * nkv // nq][:pos[i] + 1], V[l][hh * nkv // nq][:pos[i] + 1]
                    sc = kk @ q[i, hh] / math.sqrt(D)
                    p = np.exp(sc - sc.max())
                    o[i, hh] = p @ vv / p.sum()
            h = h + self.act(o.reshape(n, -1)) @ wo.T
            gu = self.act(self.norm(h, self.w[3 + 6 * l + 3])) @ wgu.T
            g, u = gu[:, :c["ffn"]], gu[:, c["ffn"]:]
            h = h + self.act(g / (1 + np.exp(-g)) * u) @ wdown.T
        a = bf16(self.norm(h, self.w[1]).astype(np.float32)).astype(np.float64)
        return a @ self.w[2].T
