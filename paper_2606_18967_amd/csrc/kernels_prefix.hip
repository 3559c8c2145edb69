// kernels_prefix.hip -- groups of sequences that share a prompt, over a paged bf16
// cache: the append that rotates and stores new rows, and the attention that reads
// the positions a group shares once for all of its rows.
//
// With the positions of a row cut into parts, each part gives m = max of the scores,
// l = sum 2^(s - m) and o = sum 2^(s - m) v (scores times log2 e), and parts join as
// l = sum l_j 2^(m_j - m), o likewise: a part may be any set of positions, so a
// group's shared ones [0, P) make parts for the rows of all its sequences together,
// and each sequence's own positions [P, kv_len + n) parts of its own.
#include <hip/hip_ext.h>
#include <limits.h>

#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "rope_rows.h"

namespace {

typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));

// the page of a slot's positions [lp P, (lp + 1) P), -1 where the block table has
// no valid one
__device__ __forceinline__ int page_of(const kv_geom& g, int slot, int lp)
{
    if (lp < 0 || lp >= g.mpp) return -1;
    const int pg = g.bt[(size_t)slot * g.mpp + lp];
    return pg >= 0 && pg < g.n_pages ? pg : -1;
}

// ------------------------------------------------------------------ append
// A work-group a row, D/8 lanes a head, U of a thread's heads under way at once: the row's
// position, page and table entries are looked up once.  Bound by the rows' bytes,
// with few rows by the chain of loads slot, length, page.
template <typename T, int D>
__global__ void __launch_bounds__(256) k_kv_append(rows_t r, kv_geom g, uint16_t* kc, uint16_t* vc, int n_q, int n_kv, kv4_src<T> xk,
                                                   kv4_src<T> xv, kv4_src<T> xq, uint16_t* q_out, kv4_rope ro)
{
    constexpr int LPR = D / 8, HPP = 256 / LPR, U = 4;             // lanes a head, heads a pass
    const int idx = blockIdx.x, b = idx / r.n, i = idx - b * r.n;
    const int nl = r.lim ? r.lim[b] : r.n, nlive = min(max(nl, 0), r.n);
    const int slot = r.slots[b];
    const bool has_slot = slot >= 0 && slot < r.max_slots, first = i == 0 && threadIdx.x == 0;
    if (first && nl != nlive) raise(r.err, ERR_LEN);
    if (i >= nlive) return;
    const int pos = has_slot ? kv4_base((long long)r.kv_len[slot] + r.off) + i : -1;
    const int stop = ro.rot ? min(r.max_ctx, ro.len) : r.max_ctx;  // first position without a table row or a place
    const bool ok = pos >= 0 && pos < stop;
    if (threadIdx.x == 0 && !ok) raise(r.err, has_slot ? ERR_CTX : ERR_SLOT);
    const int page = ok ? page_of(g, slot, pos / g.P) : -1;
    if (threadIdx.x == 0 && ok && page < 0) raise(r.err, ERR_PAGE);
    const int lw = threadIdx.x % LPR, d0 = 8 * lw, nq = q_out ? n_q : 0, units = nq + 2 * n_kv;
    float2 tr[8] = {};
    if (ok) turns(ro, pos, d0, tr);
    const long long at = (long long)max(page, 0) * g.PS + (long long)(max(pos, 0) % g.P) * D + d0;
    for (int u0 = threadIdx.x / LPR; u0 - (int)(threadIdx.x / LPR) < units; u0 += U * HPP) {
        oct<T> x[U] = {};
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int u = u0 + j * HPP;
            if (!ok || u >= units) continue;
            if (u < nq) x[j].load(xq, (size_t)idx * xq.ld + (size_t)u * D + d0);
            else if (u < nq + n_kv) x[j].load(xk, (size_t)idx * xk.ld + (size_t)(u - nq) * D + d0);
            else x[j].load(xv, (size_t)idx * xv.ld + (size_t)(u - nq - n_kv) * D + d0);
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int u = u0 + j * HPP;
            float y[8];
            // (every lane of a wave takes part: the rotation's partner may be another lane's)
            turn<float>(x[j], tr, d0, ro, y);
            if (u >= units) continue;
            if (u >= nq + n_kv) x[j].get(x[j].w, y);
            const u32x4 v = {pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])};
            if (u < nq) *(u32x4*)(q_out + ((size_t)idx * n_q + u) * D + d0) = v;
            else if (page >= 0) {
                const bool is_v = u >= nq + n_kv;
                *(u32x4*)((is_v ? vc : kc) + at + (u - nq - (is_v ? n_kv : 0)) * g.HS) = v;
            }
        }
    }
}

// ------------------------------------------------------------------ plan
// inclusive sum over the 1024 threads of a work-group; sh: 16 ints
__device__ __forceinline__ int scan1024(int v, int* sh)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(v, o, WAVE);
        if (lane >= o) v += t;
    }
    __syncthreads();
    if (lane == 63) sh[w] = v;
    __syncthreads();
    for (int i = 0; i < w; ++i) v += sh[i];
    return v;
}

__device__ __forceinline__ int cdiv(int a, int b) { return (a + b - 1) / b; }

// The items of a call (px_item): runs of sequences of one group that follow one
// another share min(len, the shortest kv_len among them) positions, rounded down to
// whole tiles; both these and the sequences' own positions are cut into chunks of
// about W / target positions, W being what all items read in all (a slice of PX_ROWS
// rows reads its chunk by itself).  Thread t is sequence t and run t.
__global__ void __launch_bounds__(1024) k_prefix_plan(rows_t r, px_groups gr, px_plan pl, int G)
{
    __shared__ int s_gid[PX_SEQS];
    __shared__ int s_first[PX_SEQS + 1], s_P[PX_SEQS], s_reader[PX_SEQS], s_live[PX_SEQS], s_rchunk[PX_SEQS], s_rend[PX_SEQS], s_rpart[PX_SEQS];
    __shared__ int s_run[PX_SEQS], s_ctx[PX_SEQS], s_ochunk[PX_SEQS], s_oend[PX_SEQS], s_opart[PX_SEQS];
    __shared__ unsigned long long s_work;
    __shared__ int sh[16], s_total[3];
    const int t = threadIdx.x, RG = r.n * G, zs = cdiv(RG, PX_ROWS);
    const bool mine = t < r.B;
    int slot = -1, nlive = 0, base = 0, gid = -1;
    bool ok = false;
    if (mine) {
        slot = r.slots[t];
        const int nl = r.lim ? r.lim[t] : r.n;
        nlive = min(max(nl, 0), r.n);
        if (nl != nlive) raise(r.err, ERR_LEN);
        if (slot >= 0 && slot < r.max_slots) {
            base = kv4_base((long long)r.kv_len[slot] + r.off);
            ok = base >= 0 && base < r.max_ctx;
            if (nlive > 0 && (base < 0 || base > r.max_ctx - nlive)) raise(r.err, ERR_CTX);
            if (ok && gr.group) {
                gid = gr.group[slot];
                if (gid < 0 || gid >= gr.n_groups) gid = -1;
            }
        } else if (nlive > 0) {
            raise(r.err, ERR_SLOT);
        }
    }
    s_gid[t] = gid;
    s_P[t] = s_reader[t] = INT_MAX;
    s_live[t] = 0;
    if (t == 0) s_work = 0;
    __syncthreads();
    // runs
    const bool lead = mine && (t == 0 || gid < 0 || gid != s_gid[t - 1]);
    const int run = scan1024(lead ? 1 : 0, sh) - 1;
    s_run[t] = run;
    if (lead) s_first[run] = t;
    if (t == r.B - 1) {
        s_first[run + 1] = r.B;
        s_total[0] = run + 1;
    }
    const bool live = ok && nlive > 0;
    __syncthreads();
    const int nruns = s_total[0];
    if (live) {
        atomicMin(&s_P[run], base);
        atomicMin(&s_reader[run], t);
        atomicAdd(&s_live[run], 1);
    }
    __syncthreads();
    int P = 0, rows = 0, slices = 0;
    if (t < nruns) {
        const int f = s_first[t], g = s_gid[f];
        rows = (s_first[t + 1] - f) * RG;
        if (g >= 0 && s_live[t] > 1) P = max(min(gr.len[g], s_P[t]), 0) / PX_TILE * PX_TILE;
        if (P > 0) slices = cdiv(rows, PX_ROWS);
    }
    __syncthreads();
    s_P[t] = P;
    __syncthreads();
    // chunks
    const int ctx = live ? min(base + nlive, r.max_ctx) : 0, pre = live ? s_P[run] : 0, own = ctx - pre;
    const unsigned long long w = (unsigned long long)P * slices + (unsigned long long)own * zs;
    if (w) atomicAdd(&s_work, w);
    __syncthreads();
    // (no context is longer than 2^24: past 2^25 nothing is cut either way)
    const int share = (int)min(max((s_work + pl.target - 1) / pl.target, (unsigned long long)pl.min_chunk), 1ull << 25);
    auto cut = [&](int x, int& chunk) {                            // chunks of x positions, as even as whole tiles allow
        if (x <= 0) return chunk = 0;
        chunk = cdiv(cdiv(x, cdiv(x, share)), PX_TILE) * PX_TILE;
        return cdiv(x, chunk);
    };
    int pchunk, ochunk;
    const int np = cut(P, pchunk), no = nlive > 0 ? max(cut(own, ochunk), 1) : 0;
    if (own <= 0) ochunk = 0;
    // a sequence that is one item writes the output itself; partial rows: the runs' first, then the sequences'
    s_live[t] = np;
    __syncthreads();
    const bool direct = no == 1 && s_live[max(run, 0)] == 0;
    const int rend = scan1024(np * slices, sh), rpart = scan1024(np * rows, sh);
    const int oend = scan1024(no * zs, sh), opart = scan1024(direct ? 0 : no * RG, sh);
    if (t == 1023) {
        s_total[0] = rend;
        s_total[1] = oend;
        s_total[2] = rpart;
    }
    s_rchunk[t] = pchunk;
    s_rend[t] = rend;
    s_rpart[t] = rpart - np * rows;
    s_ctx[t] = ctx;
    s_ochunk[t] = ochunk;
    s_oend[t] = oend;
    __syncthreads();
    s_opart[t] = direct ? -1 : s_total[2] + opart - no * RG;
    __syncthreads();
    if (mine) {
        const int f = s_first[run];
        pl.seq[t] = px_seq{s_rpart[run] + (t - f) * RG, s_live[run], (s_first[run + 1] - f) * RG, s_opart[t], direct ? 0 : no, 0};
    }
    const int n_shared = s_total[0], total = n_shared + s_total[1];
    for (int k = t; k < pl.max_items; k += 1024) {
        px_item it = {0, 0, -1, 0, 0, 0, 0, 0};                    // QR 0: no item
        if (k < total) {
            const bool shared = k < n_shared;
            const int want = shared ? k : k - n_shared;
            const int* ends = shared ? s_rend : s_oend;
            int lo = 0, hi = (shared ? nruns : r.B) - 1;           // the first whose items end past it
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                if (ends[mid] > want) hi = mid;
                else lo = mid + 1;
            }
            const int j = want - (lo ? ends[lo - 1] : 0);
            if (shared) {
                const int f = s_first[lo], qr = (s_first[lo + 1] - f) * RG, sl = cdiv(qr, PX_ROWS), c = j / sl, p0 = c * s_rchunk[lo];
                it = px_item{f * r.n, qr, r.slots[s_reader[lo]], p0, min(p0 + s_rchunk[lo], s_P[lo]), PX_SHARED, s_rpart[lo] + c * qr, j - c * sl};
            } else {
                const int c = j / zs, p0 = min((s_ctx[lo] ? s_P[s_run[lo]] : 0) + c * s_ochunk[lo], s_ctx[lo]);
                it = px_item{lo * r.n, RG, r.slots[lo], p0, min(p0 + s_ochunk[lo], s_ctx[lo]), 0, 0, j - c * zs};
                it.base = it.slot >= 0 && it.slot < r.max_slots ? kv4_base((long long)r.kv_len[it.slot] + r.off) : 0;
                it.part = s_opart[lo] < 0 ? -1 : s_opart[lo] + c * RG;
            }
        }
        pl.item[k] = it;
    }
}

// ------------------------------------------------------------------ attention
// 64 lanes x 16 bytes at base + off straight into LDS, in lane order from byte `lds` on.
// The compiler's wait counts do not see them.
__device__ __forceinline__ void row_dma16(const void* base, uint32_t off, uint32_t lds)
{
    asm volatile("global_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "{m0}"(lds) : "memory");
}

__device__ __forceinline__ float other_half_max(float v)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float other_half_sum(float v)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
__device__ __forceinline__ void px_store4(void* out, int out_t, size_t i, float4 v)
{
    if (out_t == ACT_F16) {
        const half2v a = {(_Float16)v.x, (_Float16)v.y}, b = {(_Float16)v.z, (_Float16)v.w};
        *(uint2*)((_Float16*)out + i) = make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
    } else {
        *(uint2*)((uint16_t*)out + i) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    }
}
// a pair of bf16 with what is not finite in it as 0
__device__ __forceinline__ uint32_t finite2(uint32_t x)
{
    const uint32_t lo = (x & 0x7f80u) == 0x7f80u ? 0u : x & 0xffffu, hi = (x & 0x7f800000u) == 0x7f800000u ? 0u : x & 0xffff0000u;
    return lo | hi;
}
__device__ __forceinline__ bool odd2(uint32_t x) { return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u; }

// A work-group takes an item's rows of one KV head: up to PX_ROWS query rows (a
// sequence's heads of the group side by side, position after position, sequence
// after sequence) over the positions [p0, p1).  Tiles of 64 positions go into LDS by
// DMA, the next one while one is used; each of the four waves has 32 rows, or
// with up to 64 rows two waves share 32 and take 32 positions of a tile each.
//   S^T = K Q^T by v_mfma_f32_32x32x16_bf16: a lane has row l%32 and the
//   positions 8 (i/4) + 4 (l/32) + i%4, i < 16, of 32, which in pairs of four are
//   the operand P^T of O^T += V^T P^T; V^T is read from its rows transposed
//   (ds_read_b64_tr_b16) at the same positions, so P never leaves its lane.
// A row's pieces of 16 bytes lie in LDS at piece ^ position % pieces, which lets the
// 32 lanes that read a column of pieces meet different banks.
// The softmax is online in base 2; a row's reference moves when a score passes it by
// more than 8.  Scores, sums and references are fp32; P is rounded to bf16 (2^-8
// of each).  Positions that a row does not see may hold anything: there the scores
// are replaced and values that are not finite taken as zeros; a row that sees such a
// value is NaN.
template <int D>
__global__ void __launch_bounds__(256, 2) k_prefix_attn(rows_t r, kv_geom g, const uint16_t* kc, const uint16_t* vc, int n_q, int n_kv,
                                                        const uint16_t* q, long long q_ld, float cs, px_plan pl, void* out, int out_t,
                                                        long long out_ld)
{
    constexpr int KS = D / 16, NB = D / 32, CPP = D / 8;           // k-steps of S, 32-dim blocks of O^T, 16-byte pieces of a row
    constexpr int TILE = PX_TILE * D * 2;                          // bytes of a tile's K, and of its V
    constexpr int NI = TILE / 4096;                                // a wave's DMA instructions for either
    constexpr int LDO = D + 4;                                     // LDS row stride of the merge
    __shared__ __attribute__((aligned(1024))) uint8_t s_buf[4 * TILE > 64 * LDO * 4 ? 4 * TILE : 64 * LDO * 4];
    __shared__ float2 s_ml[64];

    const int kvh = blockIdx.x;
    const px_item it = pl.item[blockIdx.y];
    const int QR = __builtin_amdgcn_readfirstlane(it.QR), z = __builtin_amdgcn_readfirstlane(it.z);
    const int q0 = z * PX_ROWS, nrows = min(QR - q0, PX_ROWS);
    if (nrows <= 0) return;
    const int row0 = __builtin_amdgcn_readfirstlane(it.row0), slot = __builtin_amdgcn_readfirstlane(it.slot);
    const int p0 = __builtin_amdgcn_readfirstlane(it.p0), base = __builtin_amdgcn_readfirstlane(it.base);
    const int part = __builtin_amdgcn_readfirstlane(it.part);
    const int G = n_q / n_kv, lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lr = lane & 31, h = lane >> 5;
    const bool wide = nrows > 64;                                  // a row tile a wave
    const int rt = wide ? w : w & 1;                               // the wave's row tile
    // what the slice's rows see ends with its last one; all of them see what the first one does
    const int seen_all = base == PX_SHARED ? INT_MAX : base + q0 / G + 1;
    const int p1 = base == PX_SHARED ? it.p1 : min(__builtin_amdgcn_readfirstlane(it.p1), base + (q0 + nrows - 1) / G + 1);
    const int pe = __builtin_amdgcn_readfirstlane(p1);

    // the lane's row: where it is, and the last position it sees (-1: it is not there)
    const int tq = q0 + 32 * rt + lr, ridx = tq / G, head = kvh * G + tq - ridx * G;
    const int ib = ridx % r.n, b = row0 / r.n + ridx / r.n;
    int lim = -1;
    bool exists = false;
    if (tq < QR) {
        exists = ib < (r.lim ? min(max(r.lim[b], 0), r.n) : r.n);
        const int sl = r.slots[b];
        if (exists && sl >= 0 && sl < r.max_slots) {
            const int pos = kv4_base((long long)r.kv_len[sl] + r.off) + ib;
            if (pos - ib >= 0 && pos < r.max_ctx) lim = pos;
        }
    }
    bf16x8 qf[KS];
    const uint32_t flip = cs < 0.f ? 0x80008000u : 0u;             // a negative scale goes into the queries' signs
    const float acs = fmaxf(fabsf(cs), 0x1p-126f);                 // (a scale of 0 leaves masked scores at -inf)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        u32x4 v = {0, 0, 0, 0};
        if (lim >= 0) v = *(const u32x4*)(q + (long long)(row0 + ridx) * q_ld + (long long)head * D + 16 * ks + 8 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] ^= flip;
        qf[ks] = __builtin_bit_cast(bf16x8, v);
    }

    // The wave's part of a tile: 16 positions of its block w/2, NI instructions of 1024 / (2 D).
    const int lp = lane / CPP, lc = lane % CPP;
    constexpr int PPI = 512 / D;                                   // positions an instruction
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)s_buf;
    const long long hb = (long long)pl.layer * g.LS + (long long)kvh * g.HS;
    const int nt = max(pe - p0 + PX_TILE - 1, 0) / PX_TILE;
    // pages of the 32-position blocks p0/32 + 128 win + ..: lane l holds l, l + 64 (-1: none, or past the end)
    int pgw[2] = {-1, -1}, kw = -(1 << 20);
    uint32_t there = 0;                                            // bit 2 (i % 2) + k: block k of tile i has a page
    auto issue = [&](int i) {
        const int blk0 = 2 * i;
        if (blk0 < kw || blk0 + 1 >= kw + 128) {
            kw = blk0;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int pos = p0 + 32 * (kw + 64 * k + lane);
                pgw[k] = pos < pe ? page_of(g, slot, pos / g.P) : -1;
                if (pos < pe && pgw[k] < 0) raise(r.err, ERR_PAGE);
            }
        }
        auto page_at = [&](int blk) {
            const int j = blk - kw, a = __builtin_amdgcn_readlane(pgw[0], j & 63), c = __builtin_amdgcn_readlane(pgw[1], j & 63);
            return j < 64 ? a : c;
        };
        const int pa = page_at(blk0), pb = page_at(blk0 + 1);
        there = (there & ~(3u << 2 * (i & 1))) | ((pa >= 0 ? 1u : 0u) | (pb >= 0 ? 2u : 0u)) << 2 * (i & 1);
        const int pg = w < 2 ? pa : pb;
        if (pg < 0) return;
        const int bs = p0 + 32 * (blk0 + (w >> 1));
        // (past the end: the last position again)
        const int last = min(bs + 31, pe - 1) - bs;
        const long long at = (long long)pg * g.PS + hb + (long long)(bs % g.P) * D;
        const uint32_t dst = ring + (i & 1) * (2 * TILE) + w * (NI * 1024);
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int row = 16 * (w & 1) + PPI * j + lp;           // in its block
            const uint32_t off = (uint32_t)(min(row, last) * D * 2 + ((lc ^ (row & (CPP - 1))) << 4));
            row_dma16(kc + at, off, dst + j * 1024);
            row_dma16(vc + at, off, dst + TILE + j * 1024);
        }
    };

    float m = -INFINITY, l = 0.f;
    floatx16 o[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[nb][i] = 0.f;

    // block k of the tile at `t`, positions from blk on
    auto block = [&](const uint8_t* t, int k, int blk, auto masked) {
        constexpr bool MASKED = decltype(masked)::value;
        const uint8_t* kt = t + (32 * k + lr) * D * 2;
        floatx16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const u32x4 kf = *(const u32x4*)(kt + (((2 * ks + h) ^ (lr & (CPP - 1))) << 4));
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf), qf[ks], s, 0, 0, 0);
        }
        if (MASKED) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (blk + 8 * (i >> 2) + 4 * h + (i & 3) > lim) s[i] = -INFINITY;
        }
        float bm = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) bm = fmaxf(bm, s[i]);
        bm = other_half_max(bm) * acs;
        const bool need = bm > m + 8.f;
        if (__builtin_amdgcn_ballot_w64(need)) {
            const float mn = need ? bm : m, corr = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= corr;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[nb][i] *= corr;
        }
        const float mn = m == -INFINITY ? 0.f : m;
        uint32_t pk[8];
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], acs, -mn)), c = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i + 1], acs, -mn));
            l += a + c;
            pk[i >> 1] = pack_bf16x2(a, c);
        }
        const uint8_t* vt = t + TILE + 32 * k * D * 2;
        if (MASKED) {
            // positions with a value that is not finite: the rows that see one are NaN
            const uint8_t* vr = vt + (lane >> 1) * D * 2 + (lane & 1) * D;
            bool odd = false;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                const u32x4 v = *(const u32x4*)(vr + 16 * c);
#pragma unroll
                for (int e = 0; e < 4; ++e) odd |= odd2(v[e]);
            }
            const uint64_t bad = __builtin_amdgcn_ballot_w64(odd);
            if (bad)
                for (int p = 0; p < 32; ++p)
                    if ((bad >> 2 * p & 3) && blk + p <= lim) l = __builtin_nanf("");
        }
        // lane l's pieces of the transposing reads: positions 4 h + l%16/4 (+ 8, + 16 st), dims 16 (l/16%2) + 4 (l%4) of a 32-dim block
        const int tr = 4 * h + ((lane & 15) >> 2), tc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), tb = (lane & 1) * 8;
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            const bf16x8 pf = __builtin_bit_cast(bf16x8, (u32x4){pk[4 * st], pk[4 * st + 1], pk[4 * st + 2], pk[4 * st + 3]});
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                auto piece = [&](int row) {
                    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) v4s*)(vt + row * D * 2 + (((4 * nb + tc) ^ (row & (CPP - 1))) << 4) + tb));
                };
                const v4s lo = piece(16 * st + tr), hi = piece(16 * st + 8 + tr);
                u32x4 vf = __builtin_bit_cast(u32x4, (v8s){lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
                if (MASKED) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) vf[e] = finite2(vf[e]);
                }
                o[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf), pf, o[nb], 0, 0, 0);
            }
        }
    };

    if (nt > 0) issue(0);
    const bool works = 32 * rt < nrows;
    for (int i = 0; i < nt; ++i) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_barrier();                                             // everyone's pieces are in, and tile i - 1 is done with
        const uint32_t have = there >> 2 * (i & 1);
        if (i + 1 < nt) issue(i + 1);
        if (!works) continue;
        const uint8_t* t = s_buf + (i & 1) * (2 * TILE);
        for (int k = wide ? 0 : w >> 1; k < 2; k += wide ? 1 : 2) {
            const int blk = p0 + PX_TILE * i + 32 * k;
            if (!(have >> k & 1)) continue;                        // no page, or past the end
            if (blk + 32 <= min(pe, seen_all)) block(t, k, blk, std::false_type());
            else block(t, k, blk, std::true_type());
        }
    }
    l = other_half_sum(l);
    if (lim < 0) m = -INFINITY, l = 0.f;                           // a row that is not there sees nothing (its o is not used)
    lds_barrier();
    if (!wide) {
        // the two waves of a row tile joined
        float* so = (float*)s_buf;
        if (w >= 2) {
            if (h == 0) s_ml[32 * rt + lr] = make_float2(m, l);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *(float4*)(so + (32 * rt + lr) * LDO + 32 * nb + 8 * j + 4 * h) =
                        make_float4(o[nb][4 * j], o[nb][4 * j + 1], o[nb][4 * j + 2], o[nb][4 * j + 3]);
        }
        __syncthreads();
        if (w >= 2) return;
        const float2 om = s_ml[32 * rt + lr];
        const float mm = fmaxf(m, om.x);
        const float fa = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mm), fb = om.x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(om.x - mm);
        m = mm;
        l = l * fa + om.y * fb;                                    // (what saw nothing has 0, or NaN)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 x = *(const float4*)(so + (32 * rt + lr) * LDO + 32 * nb + 8 * j + 4 * h);
                o[nb][4 * j] = o[nb][4 * j] * fa + x.x * fb;
                o[nb][4 * j + 1] = o[nb][4 * j + 1] * fa + x.y * fb;
                o[nb][4 * j + 2] = o[nb][4 * j + 2] * fa + x.z * fb;
                o[nb][4 * j + 3] = o[nb][4 * j + 3] * fa + x.w * fb;
            }
    }
    if (!exists) return;
    if (part >= 0) {
        const size_t pr = (size_t)kvh * pl.part_rows + part + tq;
        if (h == 0) pl.ml[pr] = make_float2(m, l);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *(float4*)(pl.o + pr * D + 32 * nb + 8 * j + 4 * h) =
                    make_float4(o[nb][4 * j], o[nb][4 * j + 1], o[nb][4 * j + 2], o[nb][4 * j + 3]);
        return;
    }
    const float rl = l == 0.f ? 0.f : 1.f / l;
    const size_t oi = (size_t)(row0 + ridx) * out_ld + (size_t)head * D;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            px_store4(out, out_t, oi + 32 * nb + 8 * j + 4 * h,
                      l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f)
                               : make_float4(o[nb][4 * j] * rl, o[nb][4 * j + 1] * rl, o[nb][4 * j + 2] * rl, o[nb][4 * j + 3] * rl));
}

// The parts of a row joined: D/4 lanes a (row, head), parts in order, eight under way
// at once.
template <int D>
__global__ void __launch_bounds__(256) k_prefix_combine(rows_t r, px_plan pl, int n_q, int n_kv, void* out, int out_t, long long out_ld)
{
    constexpr int LPR = D / 4, U = 8;
    const long long unit = (long long)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    const int G = n_q / n_kv;
    const int row = (int)(unit / n_q), head = (int)(unit - (long long)row * n_q), b = row / r.n, i = row - b * r.n, d = 4 * (threadIdx.x % LPR);
    if (b >= r.B || (r.lim && i >= r.lim[b])) return;
    const px_seq q = pl.seq[b];
    const int parts = q.pfx_n + q.own_n;
    if (parts == 0) return;                                        // the attention wrote the output
    const int kvh = head / G, t = i * G + head - kvh * G, RG = r.n * G;
    const size_t at = (size_t)kvh * pl.part_rows;
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c0 = 0; c0 < parts; c0 += U) {
        float2 ml[U];
        float4 x[U];
        float bm = m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = min(c0 + u, parts - 1), own = c - q.pfx_n;
            const size_t pr = at + (own < 0 ? q.pfx_part + c * q.pfx_rows : q.own_part + own * RG) + t;
            ml[u] = pl.ml[pr];
            x[u] = *(const float4*)(pl.o + pr * D + d);
            bm = fmaxf(bm, ml[u].x);
        }
        const float f = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - bm);
        m = bm;
        l *= f;
        o = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // a part that saw nothing has l = 0 and any o
            if (c0 + u >= parts || (ml[u].x == -INFINITY && ml[u].y == 0.f)) continue;
            const float e = ml[u].x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml[u].x - m);
            l += ml[u].y * e;
            o = make_float4(o.x + x[u].x * e, o.y + x[u].y * e, o.z + x[u].z * e, o.w + x[u].w * e);
        }
    }
    const float rl = l == 0.f ? 0.f : 1.f / l;
    px_store4(out, out_t, (size_t)row * out_ld + (size_t)head * D + d,
              l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o.x * rl, o.y * rl, o.z * rl, o.w * rl));
}

}  // namespace

// ======================================================================= launchers
template <typename T>
void launch_kv_append(const rows_t& r, const cache_t& c, int layer, int n_q, kv4_src<T> k, kv4_src<T> v, kv4_src<T> q, uint16_t* q_out,
                      const kv4_rope& ro, hipStream_t s)
{
    uint16_t *kc = (uint16_t*)c.k + layer * c.g.LS, *vc = (uint16_t*)c.v + layer * c.g.LS;
    const int blocks = r.B * r.n;
    if (c.head_dim == 128) k_kv_append<T, 128><<<blocks, 256, 0, s>>>(r, c.g, kc, vc, n_q, c.n_kv, k, v, q, q_out, ro);
    else k_kv_append<T, 64><<<blocks, 256, 0, s>>>(r, c.g, kc, vc, n_q, c.n_kv, k, v, q, q_out, ro);
}
template void launch_kv_append<float>(const rows_t&, const cache_t&, int, int, kv4_src<float>, kv4_src<float>, kv4_src<float>, uint16_t*,
                                      const kv4_rope&, hipStream_t);
template void launch_kv_append<f32_parts>(const rows_t&, const cache_t&, int, int, kv4_src<f32_parts>, kv4_src<f32_parts>,
                                          kv4_src<f32_parts>, uint16_t*, const kv4_rope&, hipStream_t);
template void launch_kv_append<uint16_t>(const rows_t&, const cache_t&, int, int, kv4_src<uint16_t>, kv4_src<uint16_t>, kv4_src<uint16_t>,
                                         uint16_t*, const kv4_rope&, hipStream_t);

// Two work-groups a CU are resident.  Every run and sequence may have one chunk more
// than its share of the target; a run's slices and a sequence's read their chunks each.
px_plan prefix_plan(int B, int n, int n_q, int n_kv)
{
    px_plan p = {};
    const long long RG = (long long)n * (n_q / n_kv);
    p.target = 512 / n_kv > 1 ? 512 / n_kv : 1;
    p.min_chunk = 128;
    const long long zs = (RG + PX_ROWS - 1) / PX_ROWS, run_slices = (B * RG + PX_ROWS - 1) / PX_ROWS + B / 2;
    p.max_items = p.target + run_slices + B * zs;
    p.part_rows = (long long)p.target * PX_ROWS + 2 * B * RG;
    return p;
}

static size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

size_t prefix_plan_bytes(const px_plan& p, int B, int n_kv, int D)
{
    return up256((size_t)B * sizeof(px_seq)) + up256((size_t)p.max_items * sizeof(px_item)) + up256((size_t)n_kv * p.part_rows * 8) +
           up256((size_t)n_kv * p.part_rows * D * 4);
}

void prefix_plan_bind(px_plan& p, void* buf, int B, int n_kv)
{
    char* c = (char*)buf;
    p.seq = (px_seq*)c;
    c += up256((size_t)B * sizeof(px_seq));
    p.item = (px_item*)c;
    c += up256((size_t)p.max_items * sizeof(px_item));
    p.ml = (float2*)c;
    c += up256((size_t)n_kv * p.part_rows * 8);
    p.o = (float*)c;
}

void launch_prefix_plan(const rows_t& r, const px_groups& g, const px_plan& p, int n_q, int n_kv, hipStream_t s)
{
    k_prefix_plan<<<1, 1024, 0, s>>>(r, g, p, n_q / n_kv);
}

template <int D>
static void prefix_attn_d(const rows_t& r, const px_plan& p, const cache_t& c, int n_q, const uint16_t* q, long long q_ld, float cs, void* out,
                          act_t out_t, long long out_ld, hipStream_t s, hipEvent_t ev0, hipEvent_t ev1)
{
    const dim3 grid(c.n_kv, p.max_items);
    const uint16_t *kc = (const uint16_t*)c.k, *vc = (const uint16_t*)c.v;
    if (ev0) hipExtLaunchKernelGGL(k_prefix_attn<D>, grid, dim3(256), 0, s, ev0, ev1, 0, r, c.g, kc, vc, n_q, c.n_kv, q, q_ld, cs, p, out, (int)out_t, out_ld);
    else k_prefix_attn<D><<<grid, 256, 0, s>>>(r, c.g, kc, vc, n_q, c.n_kv, q, q_ld, cs, p, out, (int)out_t, out_ld);
}

void launch_prefix_attention(const rows_t& r, px_plan p, const cache_t& c, int layer, int n_q, const uint16_t* q, long long q_ld, float scale,
                             void* out, act_t out_t, long long out_ld, hipStream_t s, hipEvent_t ev0, hipEvent_t ev1)
{
    p.layer = layer;
    const float cs = scale * 1.4426950408889634f;
    if (c.head_dim == 128) prefix_attn_d<128>(r, p, c, n_q, q, q_ld, cs, out, out_t, out_ld, s, ev0, ev1);
    else prefix_attn_d<64>(r, p, c, n_q, q, q_ld, cs, out, out_t, out_ld, s, ev0, ev1);
}

void launch_prefix_combine(const rows_t& r, const px_plan& p, int n_q, int n_kv, int D, void* out, act_t out_t, long long out_ld, hipStream_t s)
{
    const long long units = (long long)r.B * r.n * n_q;
    const int per = 256 / (D / 4);
    const unsigned blocks = (unsigned)((units + per - 1) / per);
    if (D == 128) k_prefix_combine<128><<<blocks, 256, 0, s>>>(r, p, n_q, n_kv, out, (int)out_t, out_ld);
    else k_prefix_combine<64><<<blocks, 256, 0, s>>>(r, p, n_q, n_kv, out, (int)out_t, out_ld);
}
