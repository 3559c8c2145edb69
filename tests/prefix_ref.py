"""A paged bf16 cache whose groups share pages, and attention over it in 64 bits, for the tests."""
import numpy as np
import torch

HALF = 2.0 ** -8                                       # half a step of bf16
E24 = 2.0 ** -24


class Batch:
    """Sequences of groups `sizes` that share `prefix` positions (a number a group) and have own[b] of their own
    before the n new rows; lens rows each.  What no row sees of the pools is NaN.  order: the batch's, by sequence."""

    def __init__(self, n_q, n_kv, D, sizes, prefix, own, n, page=64, lens=None, order=None, seed=0, layers=2, layer=1, spare=3,
                 max_ctx=None, pool_pages=None, device="cuda"):
        from paper_2606_18967_amd import sdrl
        rng = np.random.default_rng(seed)
        B = sum(sizes)
        self.n_q, self.n_kv, self.D, self.n, self.B, self.layer, self.page = n_q, n_kv, D, n, B, layer, page
        gid = np.repeat(np.arange(len(sizes)), sizes)
        prefix = np.array(prefix)
        self.base = prefix[gid] + np.array(own)
        self.lens = np.full(B, n) if lens is None else np.array(lens)
        top = int(max(self.base + self.lens.clip(0, n)).item())
        self.max_ctx = max_ctx or top
        per = -(-self.max_ctx // page)
        max_slots = B + 2
        slots = rng.permutation(max_slots)[:B]
        table = np.full((max_slots, per), -1, np.int64)
        pages = iter(rng.permutation(pool_pages or 2 * B * per + spare).tolist())
        used = []
        for g, size in enumerate(sizes):
            shared = [next(pages) for _ in range(prefix[g] // page)]
            for b in np.flatnonzero(gid == g):
                live = -(-int(self.base[b] + max(self.lens[b], 0)) // page)
                table[slots[b], :len(shared)] = shared
                rest = [next(pages) for _ in range(min(live, per) - len(shared))]
                table[slots[b], len(shared):len(shared) + len(rest)] = rest
                used += rest
            used += shared
        n_pages = pool_pages or (max(used) + 1 + spare)
        gd = torch.Generator(device=device).manual_seed(seed)
        self.k, self.v = (torch.full((n_pages, layers, n_kv, page, D), float("nan"), dtype=torch.bfloat16, device=device) for _ in range(2))
        new = lambda m: torch.randn((m, n_kv, D), generator=gd, device=device).bfloat16()  # noqa: E731
        heads = [(new(int(prefix[g])), new(int(prefix[g]))) for g in range(len(sizes))]
        self.K, self.V = [], []                        # of each sequence, [positions][n_kv][D]
        for b in range(B):
            m = int(self.base[b] - prefix[gid[b]] + max(self.lens[b], 0))
            for pool, keep, head in ((self.k, self.K, heads[gid[b]][0]), (self.v, self.V, heads[gid[b]][1])):
                x = torch.cat((head, new(m)))
                keep.append(x)
                P = np.arange(min(len(x), self.max_ctx))
                pg = torch.from_numpy(table[slots[b], P // page]).to(device)
                pool[pg, layer, :, torch.from_numpy(P % page).to(device)] = x[:len(P)]
        self.q = torch.randn((B, n, n_q, D), generator=gd, device=device).bfloat16()
        i32 = lambda a: torch.from_numpy(np.asarray(a)).to(torch.int32).to(device)  # noqa: E731
        order = np.arange(B) if order is None else np.array(order)
        self.order = order
        self.table, self.slots_h = i32(table), slots[order]
        self.slots = i32(slots[order])
        kv_len, group = np.zeros(max_slots, np.int64), np.full(max_slots, -1)
        kv_len[slots], group[slots] = self.base, gid
        self.kv_len, self.group, self.length = i32(kv_len), i32(group), i32(prefix)
        self.base, self.lens_h = self.base[order], self.lens[order]
        self.K, self.V = [self.K[b] for b in order], [self.V[b] for b in order]
        self.lens = None if lens is None else i32(self.lens_h)
        self.cache = sdrl.KVPages(self.k, self.v, self.table, self.kv_len, self.max_ctx)
        self.groups = sdrl.PrefixGroups(self.group, self.length)

    def run(self, groups=True, **kw):
        from paper_2606_18967_amd import sdrl
        out = kw.pop("out", None)
        if out is None:
            out = torch.full(self.q.shape, 7.0, dtype=torch.bfloat16, device=self.q.device)
        return sdrl.prefix_attention(self.cache, self.groups if groups else None, self.layer, self.slots, kw.pop("q", self.q), out,
                                     lens=self.lens, **kw)

    def expected(self, b, scale=None):
        """Rows of sequence b in 64 bits, [lens][n_q][D], and how far the kernel's may be off."""
        G, m = self.n_q // self.n_kv, int(self.lens_h[b])
        scale = self.D ** -0.5 if scale is None else scale
        q = self.q[b, :m].double()                                             # [m, n_q, D]
        K, V = (x.double().repeat_interleave(G, 1) for x in (self.K[b], self.V[b]))     # [P, n_q, D]
        s = torch.einsum("ihd,phd->hip", q, K) * scale
        # a score's sum of D products in fp32, and its product with scale log2 e, in units of the exponent
        ds = torch.einsum("ihd,phd->hip", q.abs(), K.abs()).amax((0, 2)) * abs(scale) * E24 * (self.D + 8)
        pos = torch.arange(len(K), device=q.device)
        seen = (pos[None] <= int(self.base[b]) + torch.arange(m, device=q.device)[:, None])[None]
        s = torch.where(seen, s, -torch.inf)
        p = torch.softmax(s, -1)
        vz = V                                                                 # (all of a sequence's own values are finite)
        o = torch.einsum("hip,phd->ihd", p, vz)
        a = torch.einsum("hip,phd->ihd", p, vz.abs())
        # P's rounding, the scores', the powers' and the sums' (a lane adds few of them); then the output's rounding
        tol = a * (HALF + 2 * ds[:, None, None] + E24 * (len(K) / 16 + 64)) + HALF * o.abs() * (1 + 2 * HALF) + 1e-30
        return o, tol

    def check(self, out, scale=None, seqs=None):
        for b in range(self.B) if seqs is None else seqs:
            m = int(self.lens_h[b])
            if m > 0:
                o, tol = self.expected(b, scale)
                off = (out[b, :m].double() - o).abs()
                assert bool((off <= tol).all()), (b, float((off / tol).max()))
            assert bool((out[b, max(m, 0):] == 7).all()), f"rows past the last of sequence {b} were written"
