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
// D/8 lanes a head.  Rows of many heads (WIDE) take a work-group each, U of a thread's heads under
// way at once: the row's position, page and table entries are looked up once.  Rows of fewer heads
// lie side by side in a work-group, a head a thread group.  Bound by the rows' bytes, short rows and few of them by
// the chain of loads slot, length, page: 12216 fp32 rows of 12 heads of 64, 28 MB, take 12.2 us (with a
// work-group each 19.0, with four rows of a thread under way 15.6), 8 rows of 48 heads of 128 4.5 us.
template <typename T, int D, bool WIDE>
__global__ void __launch_bounds__(256) k_kv_append(rows_t r, kv_geom g, uint16_t* kc, uint16_t* vc, int n_q, int n_kv, kv4_src<T> xk,
                                                   kv4_src<T> xv, kv4_src<T> xq, uint16_t* q_out, kv4_rope ro)
{
    constexpr int LPR = D / 8, HPP = 256 / LPR, U = WIDE ? 4 : 1;  // lanes a head, heads a pass
    const int nq = q_out ? n_q : 0, units = nq + 2 * n_kv, place = threadIdx.x / LPR, d0 = 8 * (threadIdx.x % LPR);
    const int abreast = WIDE ? 1 : HPP / units, sub = WIDE ? 0 : place / units, idx = blockIdx.x * abreast + sub;
    const bool in = WIDE || (sub < abreast && idx < r.B * r.n);
    const int b = in ? idx / r.n : 0, i = in ? idx - b * r.n : 0;
    const int nl = r.lim ? r.lim[b] : r.n, nlive = min(max(nl, 0), r.n), slot = r.slots[b];
    const bool there = in && i < nlive, tells = in && d0 == 0 && place == sub * units, has_slot = slot >= 0 && slot < r.max_slots;
    if (tells && i == 0 && nl != nlive) raise(r.err, ERR_LEN);
    if (WIDE && !there) return;
    const int pos = there && has_slot ? kv4_base((long long)r.kv_len[slot] + r.off) + i : -1;
    const int stop = ro.rot ? min(r.max_ctx, ro.len) : r.max_ctx;  // first position without a table row or a place
    const bool ok = pos >= 0 && pos < stop;
    if (tells && there && !ok) raise(r.err, has_slot ? ERR_CTX : ERR_SLOT);
    const int page = ok ? page_of(g, slot, pos / g.P) : -1;
    if (tells && ok && page < 0) raise(r.err, ERR_PAGE);
    float2 tr[8] = {};
    if (ok) turns(ro, pos, d0, tr);
    const long long at = (long long)max(page, 0) * g.PS + (long long)(max(pos, 0) % g.P) * D + d0;
    const int own = WIDE ? place : place - sub * units;
    for (int u0 = 0; u0 < (WIDE ? units : 1); u0 += U * HPP) {
        oct<T> x[U] = {};
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int u = own + u0 + j * HPP;
            if (!ok || u >= units) continue;
            if (u < nq) x[j].load(xq, (size_t)idx * xq.ld + (size_t)u * D + d0);
            else if (u < nq + n_kv) x[j].load(xk, (size_t)idx * xk.ld + (size_t)(u - nq) * D + d0);
            else x[j].load(xv, (size_t)idx * xv.ld + (size_t)(u - nq - n_kv) * D + d0);
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int u = own + u0 + j * HPP;
            float y[8];
            // (every lane of a wave takes part: the rotation's partner may be another lane's)
            turn<float>(x[j], tr, d0, ro, y);
            if (!there || u >= units) continue;
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
// How a call is cut into work-groups.  Sequences of one group that follow one another
// are a run; what a run shares, min(len, the shortest kv_len in it), is rounded
// down to whole tiles of PX_TILE positions.  Sequences of a run whose rows fit PX_ROWS
// make a slice (a longer sequence makes several, of PX_ROWS rows each), and a slice
// walks one stream of tiles: the shared positions, for all of its rows, then each of
// its sequences' own.  All streams are cut into chunks of about W / target tiles (W:
// the tiles of all), so that the work-groups are alike and resident at once, however
// the batch divides between shared and own positions: with items of their own for the
// sequences' tails, 8 groups of 8 behind prompts of 2048 (responses of up to 512) took
// a fifth longer, for a tail's item was 4 us of tiles and 8 of start and end.  All
// tiles count alike: an own tile of a wide slice is a wave's work, but comes from memory
// for this slice alone (counted as 2/3 of a shared one, 64 sequences behind 32768 took
// 13% longer, as 5/4 6%).

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

// inclusive sum over the lanes, by lane permutations in registers (within 16 lanes, then across)
__device__ __forceinline__ int wave_scan(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);    // from lane - 1, - 2, - 4, - 8 of a row of 16
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);    // lane 15 of the row before to rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);    // lane 31 to rows 2 and 3
    return v;
}
// the sum over the lanes of counts (whole floats)
__device__ __forceinline__ float wave_total(float v)
{
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x111, 0xf, 0xf, false));
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x112, 0xf, 0xf, false));
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x114, 0xf, 0xf, false));
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x118, 0xf, 0xf, false));
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x142, 0xa, 0xf, false));
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x143, 0xc, 0xf, false));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ int last_lane(int v) { return __builtin_amdgcn_readlane(v, 63); }
__device__ __forceinline__ int cdiv(int a, int b) { return (a + b - 1) / b; }

// What a sequence brings: where its rows are and what it may see (ctx 0: nothing), and the group it is in.
struct member { px_info info; int gid, len; };
__device__ __forceinline__ member member_of(const rows_t& r, const px_groups& gr, int b, bool report)
{
    member m = {{-1, 0, 0, 0}, -1, 0};
    const int slot = r.slots[b], nl = r.lim ? r.lim[b] : r.n, nlive = min(max(nl, 0), r.n);
    m.info.nlive = nlive;
    if (report && nl != nlive) raise(r.err, ERR_LEN);
    if (slot < 0 || slot >= r.max_slots) {
        if (report && nlive > 0) raise(r.err, ERR_SLOT);
        return m;
    }
    const int kv = r.kv_len[slot];
    if (gr.group) m.gid = gr.group[slot];
    if (m.gid < 0 || m.gid >= gr.n_groups) m.gid = -1;
    if (m.gid >= 0) m.len = gr.len[m.gid];
    const int base = kv4_base((long long)kv + r.off);
    if (report && nlive > 0 && (base < 0 || base > r.max_ctx - nlive)) raise(r.err, ERR_CTX);
    m.info.slot = slot;
    m.info.base = base;
    if (base < 0 || base >= r.max_ctx) m.gid = -1;
    else if (nlive > 0) m.info.ctx = min(base + nlive, r.max_ctx);
    return m;
}
// tiles of a sequence's own behind P shared tiles
__device__ __forceinline__ int own_tiles(const px_info& i, int P) { return i.ctx ? cdiv(i.ctx - P * PX_TILE, PX_TILE) : 0; }

// Sequences of a slice of a run of so many: alone where they share little for their rows.  A tile of few rows takes a third
// of the time of one of 128, and many slices fill the card better; what counts against them is that every slice reads
// the shared tiles.  (8 x 8 behind 256, own up to 300, 5 rows of 5 heads: alone 23 us a call, joined 30; behind 1024 36 and 37,
// behind 2048 53 and 46.  One row of 4 heads, own up to 30: behind 64 alone 15.5 and joined 15.3, behind 128 16.3 and 14.8.
// 3 rows of 4 heads, own up to 40: behind 256 18.3 and 18.3, behind 512 22.6 and 20.5.)
__device__ __forceinline__ int slice_of(const px_plan& pl, int RG, int P, int run)
{
    const int rows = min(pl.sps, run) * RG;
    return P >= max(RG / 2, rows > PX_ROWS / 2 ? 6 : 2) ? pl.sps : 1;
}

// A slice's chunks: of `tiles` tiles in shares of `share` (rows without a tile: one chunk, which writes zeros).  Slices
// of a run are cut at the same tiles, so that the shared ones, which they read at about the same time, come once
// from memory.
struct chunks { int n, len; };
// the shortest share (in tiles: one group of 8 behind 512 takes 14.2 us a call, with 1 15.1, with 3 15.1, with 4 16.4) and
// the longest, the tiles of 64 sequences of 2^24 positions
constexpr int PX_SHARE_MIN = 2, PX_SHARE_MAX = 1 << 24;
// The share is the shortest of a few that makes at most `target` items, which are then resident at once: the even one
// times 1, 9/8, .. 3/2, 2, 5/2, 3.  (8 x 8 verify rows of 5 behind 8192, two slices of 178 and 158 tiles a group and KV
// head: 135 us a call, with the even one 158; 16 x 8 behind 4096 177 and 209.)
constexpr int PX_TRIES = 8;
__device__ __forceinline__ int share_of(int even, int k) { return cdiv(even * (k < 5 ? 8 + k : 4 * k - 4), 8); }
__device__ __forceinline__ chunks chunks_of(int tiles, int share, bool any)
{
    if (!any) return {0, 0};
    if (tiles <= 0) return {1, 0};
    return {cdiv(tiles, share), min(tiles, share)};
}

// The plan of up to 64 sequences by one wave, a lane each, without a barrier: every wave of the attention makes it
// for itself where a plan kernel before it would cost more (its launch, and the way of the plan through memory).
struct wave_plan {
    px_info info;
    int P, reader, sfirst, send, nc, len, tiles, part;  // of the lane's slice: its run's shared tiles and the slot they are read through, ..
    int iend, total;                                    // items up to the lane's, and in all
};
__device__ wave_plan plan_of_wave(const rows_t& r, const px_groups& gr, const px_plan& pl, int RG, bool report)
{
    const int lane = threadIdx.x & 63;
    const bool mine = lane < r.B;
    member m = {{-1, 0, 0, 0}, -1, 0};
    if (mine) m = member_of(r, gr, lane, report);
    wave_plan p = {};
    p.info = m.info;
    const bool live = m.info.ctx > 0;
    // runs
    const int before = __shfl_up(m.gid, 1, WAVE);
    const bool lead = lane == 0 || !mine || m.gid < 0 || m.gid != before;
    const uint64_t heads = __builtin_amdgcn_ballot_w64(lead), upto = ~0ull >> (63 - lane), later = heads & ~upto;
    const int first = 63 - __builtin_clzll(heads & upto), end = min(later ? __builtin_ctzll(later) : 64, r.B);
    const uint64_t run = (~0ull >> (64 - max(end, 1))) & (~0ull << first), alive = __builtin_amdgcn_ballot_w64(live) & run;
    int low = live ? m.info.base : INT_MAX;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_down(low, o, WAVE);
        if (lane + o < end) low = min(low, t);
    }
    low = __shfl(low, first, WAVE);
    if (m.gid >= 0 && (alive & (alive - 1))) p.P = max(min(m.len, low), 0) / PX_TILE;
    p.reader = __shfl(m.info.slot, alive ? __builtin_ctzll(alive) : 0, WAVE);
    // slices
    const int per = slice_of(pl, RG, p.P, end - first);
    p.sfirst = first + (lane - first) / per * per;
    p.send = min(p.sfirst + per, end);
    const int own = own_tiles(m.info, p.P), upto_own = wave_scan(own);
    const int own_end = __shfl(upto_own, p.send - 1, WAVE), own_start = __shfl(upto_own, max(p.sfirst - 1, 0), WAVE);
    const uint64_t slice = (~0ull >> (64 - max(p.send, 1))) & (~0ull << p.sfirst);
    const bool any = (__builtin_amdgcn_ballot_w64(m.info.nlive > 0) & slice) != 0, sees = (__builtin_amdgcn_ballot_w64(live) & slice) != 0;
    p.tiles = sees ? p.P + own_end - (p.sfirst ? own_start : 0) : 0;
    const bool leads = mine && lane == p.sfirst;
    const float w = wave_total(leads ? (float)p.tiles * pl.zs : 0.f);
    const int even = (int)fminf(fmaxf(ceilf(w / (float)pl.target), (float)PX_SHARE_MIN), (float)PX_SHARE_MAX);
    int share = even;
    for (int k = 0; k < PX_TRIES; ++k) {
        const int s = share_of(even, k);
        const float rs = 1.f / (float)s;
        if (wave_total(leads && any ? fmaxf(ceilf((float)p.tiles * rs), 1.f) * pl.zs : 0.f) <= (float)pl.target) {
            share = s;
            break;
        }
    }
    const chunks c = chunks_of(p.tiles, share, any);
    p.nc = c.n;
    p.len = c.len;
    p.iend = wave_scan(leads ? c.n * pl.zs : 0);
    p.total = last_lane(p.iend);
    const int parts = leads && c.n > 1 ? c.n * (p.send - p.sfirst) * RG : 0, upto_parts = wave_scan(parts);
    p.part = __shfl(upto_parts - parts, p.sfirst, WAVE);
    return p;
}
__device__ __forceinline__ px_seq seq_of(const wave_plan& p, int RG)
{
    return px_seq{p.part + ((int)(threadIdx.x & 63) - p.sfirst) * RG, p.nc, (p.send - p.sfirst) * RG, 0};
}
// rows [128 zz, ..) of a slice's chunk c (zs 1: all of its rows)
__device__ __forceinline__ px_item make_item(const px_plan& pl, int RG, int f, int nseq, int reader, int P, int tiles, chunks ch, int part, int j)
{
    const int c = pl.zs == 1 ? j : j / pl.zs, zz = pl.zs == 1 ? 0 : j - c * pl.zs, rows = pl.zs == 1 ? nseq * RG : min(PX_ROWS, RG - PX_ROWS * zz);
    const int t0 = c * ch.len;
    return px_item{f, nseq, PX_ROWS * zz, rows, reader, P, t0, min(t0 + ch.len, tiles), ch.n > 1 ? part + zz * ch.n * PX_ROWS + c * rows : -1};
}
// item k (the same in every lane)
__device__ px_item item_of(const wave_plan& p, const px_plan& pl, int RG, int k)
{
    if (k >= p.total) return px_item{};
    const int L = __builtin_ctzll(__builtin_amdgcn_ballot_w64(p.iend > k));
    auto of = [&](int v) { return __builtin_amdgcn_readlane(v, L); };
    return make_item(pl, RG, L, of(p.send) - L, of(p.reader), of(p.P), of(p.tiles), chunks{of(p.nc), of(p.len)}, of(p.part),
                     k - (L ? __builtin_amdgcn_readlane(p.iend, L - 1) : 0));
}
// (the first wave makes the plan, every thread an item)
__global__ void __launch_bounds__(256) k_prefix_plan_wave(rows_t r, px_groups gr, px_plan pl, int RG)
{
    __shared__ int s_send[64], s_reader[64], s_P[64], s_tiles[64], s_nc[64], s_len[64], s_part[64], s_iend[64];
    const int t = threadIdx.x;
    if (t < 64) {
        const wave_plan p = plan_of_wave(r, gr, pl, RG, true);
        if (t < r.B) {
            pl.seq[t] = seq_of(p, RG);
            pl.info[t] = p.info;
        }
        s_send[t] = p.send;
        s_reader[t] = p.reader;
        s_P[t] = p.P;
        s_tiles[t] = p.tiles;
        s_nc[t] = p.nc;
        s_len[t] = p.len;
        s_part[t] = p.part;
        s_iend[t] = p.iend;
    }
    __syncthreads();
    for (int k = t; k < pl.max_items; k += 256) {
        px_item it = {};
        if (k < s_iend[63]) {
            int L = 0;                                             // the first whose items end past it
#pragma unroll
            for (int o = 32; o > 0; o >>= 1)
                if (s_iend[L + o - 1] <= k) L += o;
            it = make_item(pl, RG, L, s_send[L] - L, s_reader[L], s_P[L], s_tiles[L], chunks{s_nc[L], s_len[L]}, s_part[L], k - (L ? s_iend[L - 1] : 0));
        }
        pl.item[k] = it;
    }
}

// The same for up to PX_SEQS sequences, a thread each.
__global__ void __launch_bounds__(1024) k_prefix_plan(rows_t r, px_groups gr, px_plan pl, int RG)
{
    __shared__ int s_gid[PX_SEQS], s_first[PX_SEQS + 1], s_low[PX_SEQS], s_reader[PX_SEQS], s_alive[PX_SEQS];   // of runs, but the first
    __shared__ int s_own[PX_SEQS], s_any[PX_SEQS], s_send[PX_SEQS], s_iend[PX_SEQS], s_part[PX_SEQS], s_tiles[PX_SEQS], s_nc[PX_SEQS], s_len[PX_SEQS];
    __shared__ unsigned long long s_work;
    __shared__ int s_items[PX_TRIES];
    __shared__ int sh[16];
    const int t = threadIdx.x;
    const bool mine = t < r.B;
    member m = {{-1, 0, 0, 0}, -1, 0};
    if (mine) {
        m = member_of(r, gr, t, true);
        pl.info[t] = m.info;
    }
    const bool live = m.info.ctx > 0;
    s_gid[t] = m.gid;
    s_low[t] = s_reader[t] = INT_MAX;
    s_alive[t] = 0;
    if (t == 0) s_work = 0;
    if (t < PX_TRIES) s_items[t] = 0;
    __syncthreads();
    const bool lead = mine && (t == 0 || m.gid < 0 || m.gid != s_gid[t - 1]);
    const int run = max(scan1024(lead ? 1 : 0, sh) - 1, 0);
    if (lead) s_first[run] = t;
    if (t == r.B - 1) s_first[run + 1] = r.B;
    if (live) {
        atomicMin(&s_low[run], m.info.base);
        atomicMin(&s_reader[run], t);
        atomicAdd(&s_alive[run], 1);
    }
    __syncthreads();
    const int first = s_first[run], end = s_first[run + 1];
    const int P = m.gid >= 0 && s_alive[run] > 1 ? max(min(m.len, s_low[run]), 0) / PX_TILE : 0;
    const int per = slice_of(pl, RG, P, end - first), sfirst = first + (t - first) / per * per, send = min(sfirst + per, end);
    s_own[t] = scan1024(own_tiles(m.info, P), sh);
    s_any[t] = scan1024((m.info.nlive > 0 ? 1 << 16 : 0) + (live ? 1 : 0), sh);
    s_send[t] = send;
    __syncthreads();
    const bool leads = mine && t == sfirst;
    int tiles = 0;
    bool any = false;
    if (leads) {
        const int counts = s_any[send - 1] - (t ? s_any[t - 1] : 0);
        any = counts >> 16;
        tiles = counts & 0xffff ? P + s_own[send - 1] - (t ? s_own[t - 1] : 0) : 0;
        atomicAdd(&s_work, (unsigned long long)tiles * pl.zs);
    }
    __syncthreads();
    const int even = (int)min(max((s_work + pl.target - 1) / pl.target, (unsigned long long)PX_SHARE_MIN), (unsigned long long)PX_SHARE_MAX);
    if (leads && any)
        for (int k = 0; k < PX_TRIES; ++k) atomicAdd(&s_items[k], max(cdiv(tiles, share_of(even, k)), 1) * pl.zs);
    __syncthreads();
    int share = even;
    for (int k = PX_TRIES - 1; k >= 0; --k)
        if (s_items[k] <= pl.target) share = share_of(even, k);
    const chunks c = leads ? chunks_of(tiles, share, any) : chunks{0, 0};
    s_iend[t] = scan1024(c.n * pl.zs, sh);
    const int parts = c.n > 1 ? c.n * (send - sfirst) * RG : 0;
    s_part[t] = scan1024(parts, sh) - parts;
    s_tiles[t] = tiles;
    s_nc[t] = c.n;
    s_len[t] = c.len;
    __syncthreads();
    if (mine) pl.seq[t] = px_seq{s_part[sfirst] + (t - sfirst) * RG, s_nc[sfirst], (send - sfirst) * RG, 0};
    s_low[t] = P;                                                  // (of the runs before, from here on of the sequences)
    if (mine) s_gid[t] = s_reader[run] < r.B ? r.slots[s_reader[run]] : -1;
    __syncthreads();
    for (int k = t; k < pl.max_items; k += 1024) {
        px_item it = {};
        if (k < s_iend[1023]) {
            int L = 0;
#pragma unroll
            for (int o = 512; o > 0; o >>= 1)
                if (s_iend[L + o - 1] <= k) L += o;
            it = make_item(pl, RG, L, s_send[L] - L, s_gid[L], s_low[L], s_tiles[L], chunks{s_nc[L], s_len[L]}, s_part[L], k - (L ? s_iend[L - 1] : 0));
        }
        pl.item[k] = it;
    }
}

// ------------------------------------------------------------------ attention
typedef __attribute__((address_space(3))) uint8_t* lds_t;
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

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

// Up to a reference of this size a score leaves it as one fused operation with the scale: that is exact but for the reference's own
// rounding, which all of a row's weights have in common (2^0.5 at most).  Past it the scores are rounded as the reference was,
// before they leave it: what rounding leaves between the two would be of any size (2^128 from scores of 2^31 on).
constexpr float PX_FUSED = 0x1p24f;

template <int D>
__device__ __forceinline__ constexpr int v_swizzle(int row) { return D == 128 ? (row & 3) << 2 : (row & 2) << 1; }

// A work-group takes a slice's rows of one KV head, up to PX_ROWS (a sequence's heads of
// the group side by side, position after position, sequence after sequence), over the
// tiles [t0, t1) of its stream.  Tiles of 64 positions go into LDS by DMA, the next
// one while one is used; each of the four waves has 32 rows, or with up to 64 rows
// two waves share 32 and take 32 positions of a tile each.
//   S^T = K Q^T by v_mfma_f32_32x32x16_bf16: a lane has row l%32 and the
//   positions 8 (i/4) + 4 (l/32) + i%4, i < 16, of 32, which in pairs of four are
//   the operand P^T of O^T += V^T P^T; V^T is read from its rows transposed
//   (ds_read_b64_tr_b16) at the same positions, so P never leaves its lane.
// A K row's pieces of 16 bytes lie in LDS at piece ^ position % pieces, which lets the
// lanes that read a column of pieces meet different banks; a V row's at piece ^
// v_swizzle, for 32 lanes that read four pieces of four rows.  (With V as K its
// reads met 59% of their cycles in the same banks.)
// The softmax is online in base 2; a row's reference moves when a score passes it by
// more than 8.  Scores, sums and references are fp32; P is rounded to bf16 (2^-8
// of each).  Positions that a row does not see may hold anything: there the scores
// are replaced and values that are not finite taken as zeros; a row that sees such a
// value is NaN.
// Few rows are bound by HBM: 8 groups of 8 behind prompts of 2048 (135 MB) take 37 us, 35
// with a plan made before, 33 of them without the products.  Many are bound by the products, the softmax between them and
// the tiles' way into LDS nearly alike: 64 sequences behind 32768 positions (202 MB, 35
// GFLOP) take 65 us, 55 with all tiles from one page, 55 without the products; 8 x 8 verify
// rows of 5 behind 8192 (32B shape) 125 us, 114 and 105, and 150 once the power limit has
// lowered the clock.
// NBLK: the blocks of a tile that a wave takes, 2 with a row tile a wave
template <int D, int NBLK>
__device__ __forceinline__ void attend_item(uint8_t* s_buf, float2* s_ml, uint32_t* s_odd, const px_item& it, const px_info& inf, const rows_t& r,
                                            const kv_geom& g, const uint16_t* kc, const uint16_t* vc, int n_q, int n_kv, const uint16_t* q,
                                            long long q_ld, float cs, const px_plan& pl, void* out, int out_t, long long out_ld)
{
    constexpr int KS = D / 16, NB = D / 32, CPP = D / 8;           // k-steps of S, 32-dim blocks of O^T, 16-byte pieces of a row
    constexpr int TILE = PX_TILE * D * 2, BLOCK = TILE / 2;        // bytes of a tile's K, and of its V, and of half of it
    constexpr int NI = TILE / 4096, PPI = 512 / D;                 // a wave's DMA instructions for either, and the positions of one
    constexpr int LDO = D + 4;                                     // LDS row stride of the merge
    constexpr bool wide = NBLK == 2;
    auto uni = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    const int kvh = blockIdx.x, f = uni(it.f), nseq = uni(it.nseq), r0 = uni(it.r0), nrows = uni(it.rows), P = uni(it.P);
    const int t0 = uni(it.t0), nt = uni(it.t1) - t0, part = uni(it.part);
    const int G = n_q / n_kv, RG = r.n * G, lane = threadIdx.x & 63, w = uni(threadIdx.x >> 6), lr = lane & 31, h = lane >> 5;
    const int rt = wide ? w : w & 1;                               // the wave's row tile

    // The stream: tiles [0, P) are shared, then come `own` of each sequence.  Lane l of a window holds block l % 2 of its tile
    // l / 2: its page (-1: none, or past the end), its tile's first position, the end, and the sequence (-1: shared).
    const int own = own_tiles(inf, P), upto = wave_scan(own);
    int wpage = -1, wpos = 0, wend = 0, wseq = -1, kw = 0;
    auto window = [&] {
        const int t = t0 + kw + (lane >> 1), u = t - P;
        int s = 0;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1)
            if (__shfl(upto, s + o - 1, WAVE) <= u) s += o;
        s = min(s, 63);
        const int start = __shfl(upto - own, s, WAVE), slot = __shfl(inf.slot, s, WAVE), ctx = __shfl(inf.ctx, s, WAVE);
        const bool shared = t < P;
        wpos = shared ? t * PX_TILE : (P + u - start) * PX_TILE;
        wend = shared ? P * PX_TILE : ctx;
        wseq = shared ? -1 : s;
        const int pos = wpos + 32 * (lane & 1);
        wpage = -1;
        if (t < t0 + nt && pos < wend) {
            wpage = page_of(g, shared ? it.reader : slot, pos / g.P);
            if (wpage < 0) raise(r.err, ERR_PAGE);
        }
    };
    window();

    // the lane's row: its sequence in the slice, where it is, and the last position it sees (-1: it is not there)
    const int tq = 32 * rt + lr, sr = pl.zs == 1 ? tq / RG : 0, tt = pl.zs == 1 ? tq - sr * RG : r0 + tq, ri = tt / G, head = kvh * G + tt - ri * G;
    const int row = (f + sr) * r.n + ri, rbase = __shfl(inf.base, min(sr, 63), WAVE), rctx = __shfl(inf.ctx, min(sr, 63), WAVE);
    const int rlive = __shfl(inf.nlive, min(sr, 63), WAVE);
    const bool exists = tq < nrows && ri < rlive;
    const int lim = exists && rctx > 0 && rbase + ri < r.max_ctx ? rbase + ri : -1;

    struct tile_t { int pos, end, seq; uint32_t have; };           // have: bit k: block k has a page and positions
    const int lp = lane / CPP, lc = lane % CPP;
    const lds_t lds = (lds_t)s_buf;
    const uint32_t ring = (uint32_t)(uintptr_t)lds;
    const long long hb = (long long)pl.layer * g.LS + (long long)kvh * g.HS;
    // tile i on its way into its place in LDS: a wave takes 16 positions, past the end the last one again
    auto issue = [&](int i) {
        if (i >= kw + 32) {
            kw = i;
            window();
        }
        const int j = 2 * (i - kw), pa = __builtin_amdgcn_readlane(wpage, j), pb = __builtin_amdgcn_readlane(wpage, j + 1);
        const tile_t t = {__builtin_amdgcn_readlane(wpos, j), __builtin_amdgcn_readlane(wend, j), __builtin_amdgcn_readlane(wseq, j),
                          (pa >= 0 ? 1u : 0u) | (pb >= 0 ? 2u : 0u)};
        const int pg = w < 2 ? pa : pb;
        if (pg < 0) return t;
        const int bs = t.pos + 32 * (w >> 1), last = min(bs + 31, t.end - 1) - bs;
        const long long at = (long long)pg * g.PS + hb + (long long)(bs % g.P) * D;
        const uint32_t dst = ring + (i & 1) * (2 * TILE) + w * (NI * 1024);
#pragma unroll
        for (int k = 0; k < NI; ++k) {
            const int rr = 16 * (w & 1) + PPI * k + lp;            // in its block
            const uint32_t from = (uint32_t)(min(rr, last) * D * 2);
            row_dma16(kc + at, from + ((lc ^ (rr & (CPP - 1))) << 4), dst + k * 1024);
            row_dma16(vc + at, from + ((lc ^ v_swizzle<D>(rr)) << 4), dst + TILE + k * 1024);
        }
        return t;
    };
    tile_t next = {0, 0, -1, 0};
    if (nt > 0) next = issue(0);                                   // under way while the queries are read

    bf16x8 qf[KS];
    const uint32_t flip = cs < 0.f ? 0x80008000u : 0u;             // a negative scale goes into the queries' signs
    const float acs = fmaxf(fabsf(cs), 0x1p-126f);                 // (a scale of 0 leaves masked scores at -inf)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        u32x4 v = {0, 0, 0, 0};
        if (lim >= 0) v = *(const u32x4*)(q + (long long)row * q_ld + (long long)head * D + 16 * ks + 8 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] ^= flip;
        qf[ks] = __builtin_bit_cast(bf16x8, v);
    }

    float m = lim < 0 ? 0.f : -INFINITY, l = 0.f;                  // (a row that is not there never moves its reference)
    floatx16 o[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[nb][i] = 0.f;

    // LDS addresses from a block on: of the lane's K pieces (k-step ks at ^ 32 ks), and of its pieces of the transposing
    // reads, positions 4 h + l%16/4, dims 16 (l/16%2) + 4 (l%4) of a 32-dim block nb (at ^ 64 nb)
    const int tr = 4 * h + ((lane & 15) >> 2), tc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    const uint32_t ka = lr * D * 2 + ((h ^ (lr & (CPP - 1))) << 4), va = tr * D * 2 + ((tc ^ v_swizzle<D>(tr)) << 4) + (lane & 1) * 8;

    // The scores of the blocks whose K lies `tile` bytes into LDS.  (Left to itself the compiler reads each operand from LDS
    // right before its product, and every product waits for its read.)
    auto scores = [&](uint32_t tile, auto& s) {
        constexpr int N = sizeof(s) / sizeof(floatx16);
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[n][i] = 0.f;
        auto fetch = [&](int k) { return *(const __attribute__((address_space(3))) u32x4*)(lds + ((ka + tile) ^ (k / N * 32)) + k % N * BLOCK); };
        u32x4 kf[KS * N];
        constexpr int AHEAD = KS;                                  // reads run so many products in front of theirs
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) kf[k] = fetch(k);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < KS * N; ++k) {
            s[k % N] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[k]), qf[k / N], s[k % N], 0, 0, 0);
            if (k + AHEAD < KS * N) kf[k + AHEAD] = fetch(k + AHEAD);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // the row's largest score, in base 2
    auto top_of = [&](const auto& s) {
        constexpr int N = sizeof(s) / sizeof(floatx16);
        float bm = s[0][0];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) bm = fmaxf(bm, s[n][i]);
        return other_half_max(bm) * acs;
    };
    // The probabilities 2^(s by - from) above the reference, into l, and their products with the values `tile` bytes into LDS,
    // in an order of my own: a block's values are read while its powers are made, a second block's powers go between the first one's products.
    // cap: +inf, or -inf for a row that sees none of them (whatever its scores are).
    auto add = [&](uint32_t tile, const auto& s, float by, float from, auto capped, float cap) {
        constexpr int N = sizeof(s) / sizeof(floatx16), P = 2 * NB;    // products a block
        uint32_t pk[N][8];
        bf16x8 vf[N][P];
        auto power2 = [&](int n, int i) {                          // two of a lane's 16 probabilities
            float a = __builtin_fmaf(s[n][i], by, -from), c = __builtin_fmaf(s[n][i + 1], by, -from);
            if (decltype(capped)::value) a = fminf(a, cap), c = fminf(c, cap);
            a = __builtin_amdgcn_exp2f(a);
            c = __builtin_amdgcn_exp2f(c);
            l += a + c;
            pk[n][i >> 1] = pack_bf16x2(a, c);
        };
        auto fetch = [&](int n, int k) {                           // the operand of product k: positions 16 (k / NB), dims 32 (k % NB)
            auto piece = [&](uint32_t at) {
                return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(lds + at));
            };
            const uint32_t at = ((va + tile) ^ (k % NB * 64)) + (32 * n + 16 * (k / NB)) * D * 2;
            const v4s lo = piece(at), hi = piece(at + 8 * D * 2);
            vf[n][k] = __builtin_bit_cast(bf16x8, (v8s){lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
        };
        auto product = [&](int n, int k) {
            const int st = k / NB;
            const bf16x8 pf = __builtin_bit_cast(bf16x8, (u32x4){pk[n][4 * st], pk[n][4 * st + 1], pk[n][4 * st + 2], pk[n][4 * st + 3]});
            o[k % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[n][k], pf, o[k % NB], 0, 0, 0);
        };
#pragma unroll
        for (int k = 0; k < P; ++k) fetch(0, k);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 16; i += 2) power2(0, i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int k = 0; k < P; ++k) {
                product(n, k);
                if (n + 1 < N) {
                    fetch(n + 1, k);
#pragma unroll
                    for (int i = 0; i < 16 / P; i += 2) power2(n + 1, 16 / P * k + i);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
    };
    // A block that some row does not see (a row sees its positions from blk up to `to`), whose scores move a reference, or with
    // a reference past PX_FUSED.
    auto slow_block = [&](uint32_t tile, int blk, int to, uint32_t odd) {
        floatx16 s[1];
        scores(tile, s);
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (blk + 8 * (i >> 2) + 4 * h + (i & 3) > to) s[0][i] = -INFINITY;
        const float bm = top_of(s);
        m = m == -INFINITY ? bm : m;                               // nothing seen so far: nothing to rescale
        const bool need = bm > m + 8.f;
        if (__builtin_amdgcn_ballot_w64(need)) {
            const float corr = need ? __builtin_amdgcn_exp2f(m - bm) : 1.f;   // (a row that saw nothing yet has m = -inf)
            m = need ? bm : m;
            l *= corr;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[nb][i] *= corr;
        }
        // the rows that see a value that is not finite are NaN
        if (odd)
            for (int p = 0; p < 32; ++p)
                if ((odd >> p & 1) && blk + p <= to) l = __builtin_nanf("");
        const float ref = m == -INFINITY ? 0.f : m;
        float by = acs;
        if (fabsf(ref) > PX_FUSED) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[0][i] *= acs;
            by = 1.f;
        }
        asm volatile("" : "+v"(by));                               // (a known 1 would let the compiler fuse the two again)
        add(tile + TILE, s, by, ref, std::false_type(), 0.f);
    };
    // Values that are not finite in the wave's own 16 positions of a tile become zeros, which 0 times nothing of them is left,
    // and the positions' bits are noted for the rows that see them.  (Of a block without a page this is what lies there,
    // for nobody.)
    auto clean = [&](int i) {
        constexpr int RPP = 1024 / D / 2;                          // rows a pass, D / 8 lanes of 16 bytes each
        uint32_t odd = 0;
#pragma unroll
        for (int t = 0; t < 16 / RPP; ++t) {
            const lds_t p = lds + (i & 1) * (2 * TILE) + TILE + w * (NI * 1024) + t * 1024 + 16 * lane;
            u32x4 x = *(const __attribute__((address_space(3))) u32x4*)p;
            u16x2 most = {0, 0};
#pragma unroll
            for (int e = 0; e < 4; ++e) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, x[e] & 0x7fff7fffu));
            const bool hit = most[0] >= 0x7f80 || most[1] >= 0x7f80;
            const uint64_t b = __builtin_amdgcn_ballot_w64(hit);
            if (!b) continue;
            if (hit) {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = finite2(x[e]);
                *(__attribute__((address_space(3))) u32x4*)p = x;
            }
            for (int e = 0; e < RPP; ++e) odd |= (b >> CPP * e & (CPP == 8 ? 255 : 65535) ? 1u : 0u) << (RPP * t + e);
        }
        if (lane == 0) ((uint16_t*)s_odd)[4 * (i & 1) + w] = (uint16_t)odd;
    };

    // The walk.  Tiles are of three kinds: what every row sees as a whole, what the rows of one sequence see as a whole and the
    // others not at all, and the rest.  The first two, as long as they move no reference and find none past PX_FUSED, are loops
    // of their own, which change no sum but by adding: with the references' rescaling inside them the compiler keeps a second
    // copy of O and moves it every tile.
    enum { ALL, ONE, PART };
    const bool works = 32 * rt < nrows;
    const int from = wide ? 0 : w >> 1, first_row = r0 / G;        // the wave's first block, the slice's first row of its sequence
    constexpr uint32_t mine = wide ? 3 : 1;
    tile_t cur = next;
    uint32_t have = 0;
    int i = -1, kind = PART;
    bool dirty = false;                                            // tile i was cleaned
    // the next tile in which the wave has something to do; false: there is none
    auto advance = [&] {
        while (++i < nt) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            cur = next;
            const bool whole = cur.seq < 0 || cur.pos + PX_TILE <= min(cur.end, __builtin_amdgcn_readlane(inf.base, cur.seq & 63) + first_row + 1);
            const bool one = cur.seq >= 0 && nseq > 1;
            dirty = one || !whole;
            if (dirty) clean(i);
            lds_barrier();                                         // everyone's pieces are in, and tile i - 1 is done with
            if (i + 1 < nt) next = issue(i + 1);
            have = cur.have >> from & mine;
            kind = !whole || have != mine ? PART : one ? ONE : ALL;
            if (works && have && (!dirty || __builtin_amdgcn_ballot_w64(sr == cur.seq && lim >= cur.pos))) return true;
        }
        return false;
    };
    for (bool more = true; advance();) {
        const auto walk = [&](auto which) {
            constexpr int KIND = decltype(which)::value;
            while (more && kind == KIND) {
                const uint32_t tile = (i & 1) * (2 * TILE) + BLOCK * from;
                floatx16 s[NBLK];
                scores(tile, s);
                float top = top_of(s), cap = INFINITY;
                if (KIND == ONE) {
                    if (sr != cur.seq) top = cap = -INFINITY;
                    uint32_t odd = 0;
                    for (int n = 0; n < NBLK; ++n) odd |= s_odd[2 * (i & 1) + from + n];
                    if (odd && sr == cur.seq) l = __builtin_nanf("");
                }
                m = m == -INFINITY ? top : m;                      // nothing seen so far: nothing to rescale
                const float ref = m == -INFINITY ? 0.f : m;
                if (__builtin_amdgcn_ballot_w64(top > m + 8.f || fabsf(ref) > PX_FUSED)) {
                    kind = PART;
                    return;
                }
                add(tile + TILE, s, acs, ref, std::integral_constant<bool, KIND == ONE>(), cap);
                more = advance();
            }
        };
        walk(std::integral_constant<int, ALL>());
        walk(std::integral_constant<int, ONE>());
        if (!more) break;
        // (of a shared tile, or of a slice's only sequence, rows may be compared with any position that they see)
        const int to = cur.seq < 0 ? INT_MAX : sr == cur.seq ? lim : -1;
#pragma clang loop unroll(disable)
        for (int n = 0; n < NBLK; ++n)
            if (have >> n & 1)
                slow_block((i & 1) * (2 * TILE) + BLOCK * (from + n), cur.pos + 32 * (from + n), to, dirty ? s_odd[2 * (i & 1) + from + n] : 0);
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
    const size_t oi = (size_t)row * out_ld + (size_t)head * D;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            px_store4(out, out_t, oi + 32 * nb + 8 * j + 4 * h,
                      l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f)
                               : make_float4(o[nb][4 * j] * rl, o[nb][4 * j + 1] * rl, o[nb][4 * j + 2] * rl, o[nb][4 * j + 3] * rl));
}

// SELF: without a plan in memory, it is made here
template <int D, bool SELF>
__global__ void __launch_bounds__(256, 2) k_prefix_attn(rows_t r, kv_geom g, const uint16_t* kc, const uint16_t* vc, int n_q, int n_kv,
                                                        const uint16_t* q, long long q_ld, float cs, px_plan pl, px_groups gr, void* out,
                                                        int out_t, long long out_ld)
{
    constexpr int RING = 4 * PX_TILE * D * 2, MERGE = 64 * (D + 4) * 4;
    __shared__ __attribute__((aligned(1024))) uint8_t s_buf[RING > MERGE ? RING : MERGE];
    __shared__ float2 s_ml[64];
    __shared__ uint32_t s_odd[4];                                  // of the ring's two tiles, a bit a position
    const int lane = threadIdx.x & 63;
    px_item it;
    px_info inf = {-1, 0, 0, 0};                                   // lane l: of the slice's sequence l
    if constexpr (SELF) {
        const bool teller = blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 64;
        const int RG = r.n * (n_q / n_kv);
        const wave_plan p = plan_of_wave(r, gr, pl, RG, teller);
        if (teller && lane < r.B) pl.seq[lane] = seq_of(p, RG);
        it = item_of(p, pl, RG, blockIdx.y);
        const int at = min(it.f + lane, 63);
        const px_info x = {__shfl(p.info.slot, at, WAVE), __shfl(p.info.base, at, WAVE), __shfl(p.info.ctx, at, WAVE), __shfl(p.info.nlive, at, WAVE)};
        if (lane < it.nseq) inf = x;
    } else {
        it = pl.item[blockIdx.y];
        if (lane < it.nseq) inf = pl.info[it.f + lane];
    }
    const int rows = __builtin_amdgcn_readfirstlane(it.rows);
    if (rows == 0) return;                                         // no item
    if (rows > 64) attend_item<D, 2>(s_buf, s_ml, s_odd, it, inf, r, g, kc, vc, n_q, n_kv, q, q_ld, cs, pl, out, out_t, out_ld);
    else attend_item<D, 1>(s_buf, s_ml, s_odd, it, inf, r, g, kc, vc, n_q, n_kv, q, q_ld, cs, pl, out, out_t, out_ld);
}

// Two sums of parts made one: the references, sums and four of the dims.
struct px_sum { float m, l; float4 o; };
__device__ __forceinline__ px_sum both(const px_sum& a, const px_sum& b)
{
    const float m = fmaxf(a.m, b.m);
    const float fa = a.m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(a.m - m), fb = b.m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(b.m - m);
    return {m, a.l * fa + b.l * fb,
            make_float4(a.o.x * fa + b.o.x * fb, a.o.y * fa + b.o.y * fb, a.o.z * fa + b.o.z * fb, a.o.w * fa + b.o.w * fb)};
}

// The parts of a row joined: W waves a (row, head), D/4 lanes a part, U parts of each under way at once; a
// part that saw nothing of the row is not read.  Bound by the parts' bytes and, with few, by its launch: 64 rows of 32
// heads in 32 parts (34 MB) take 8 us, 8 rows of 32 heads in 20 parts 4.
template <int D, int W>
__global__ void __launch_bounds__(256) k_prefix_combine(rows_t r, px_plan pl, int n_q, int n_kv, void* out, int out_t, long long out_ld)
{
    constexpr int LPP = D / 4, NP = WAVE / LPP, U = 4;             // lanes a part, parts side by side
    __shared__ px_sum s_sum[W > 1 ? W : 1][LPP];
    const int w = W > 1 ? threadIdx.x >> 6 : 0;
    const long long unit = W > 1 ? blockIdx.x : (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int G = n_q / n_kv, row = (int)(unit / n_q), head = (int)(unit - (long long)row * n_q), b = row / r.n, i = row - b * r.n;
    if (b >= r.B || (r.lim && i >= r.lim[b])) return;
    const px_seq q = pl.seq[b];
    if (q.nc <= 1) return;                                         // the attention wrote the output
    const int lane = threadIdx.x & 63, d = 4 * (lane % LPP), side = lane / LPP;
    const int kvh = head / G, t = i * G + head - kvh * G, RG = r.n * G, zz = pl.zs == 1 ? 0 : t / PX_ROWS;
    const int stride = pl.zs == 1 ? q.stride : min(PX_ROWS, RG - PX_ROWS * zz);
    const size_t at = (size_t)kvh * pl.part_rows + q.part + (size_t)zz * q.nc * PX_ROWS + (t - PX_ROWS * zz);
    px_sum s = {-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
    for (int c0 = w * NP + side; c0 < q.nc; c0 += U * W * NP) {
        float2 ml[U];
        float4 x[U];
        float bm = s.m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            ml[u] = make_float2(-INFINITY, 0.f);
            if (c0 + u * W * NP < q.nc) ml[u] = pl.ml[at + (size_t)(c0 + u * W * NP) * stride];
            bm = fmaxf(bm, ml[u].x);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (ml[u].x != -INFINITY || ml[u].y != 0.f) x[u] = *(const float4*)(pl.o + (at + (size_t)(c0 + u * W * NP) * stride) * D + d);
        }
        const float f = s.m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(s.m - bm);
        s = {bm, s.l * f, make_float4(s.o.x * f, s.o.y * f, s.o.z * f, s.o.w * f)};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float e = ml[u].x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml[u].x - bm);
            s.l += ml[u].y * e;
            s.o = make_float4(s.o.x + x[u].x * e, s.o.y + x[u].y * e, s.o.z + x[u].z * e, s.o.w + x[u].w * e);
        }
    }
    // the sides joined, in all of them alike, then the waves
#pragma unroll
    for (int k = LPP; k < WAVE; k <<= 1)
        s = both(s, px_sum{__shfl_xor(s.m, k, WAVE), __shfl_xor(s.l, k, WAVE),
                           make_float4(__shfl_xor(s.o.x, k, WAVE), __shfl_xor(s.o.y, k, WAVE), __shfl_xor(s.o.z, k, WAVE), __shfl_xor(s.o.w, k, WAVE))});
    if (W > 1) {
        if (side == 0) s_sum[w][lane] = s;
        __syncthreads();
        if (w) return;
        s = s_sum[0][lane % LPP];
#pragma unroll
        for (int k = 1; k < W; ++k) s = both(s, s_sum[k][lane % LPP]);
    }
    if (side) return;
    const float rl = s.l == 0.f ? 0.f : 1.f / s.l;
    px_store4(out, out_t, (size_t)row * out_ld + (size_t)head * D + d,
              s.l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(s.o.x * rl, s.o.y * rl, s.o.z * rl, s.o.w * rl));
}

}  // namespace

// ======================================================================= launchers
template <typename T>
void launch_kv_append(const rows_t& r, const cache_t& c, int layer, int n_q, kv4_src<T> k, kv4_src<T> v, kv4_src<T> q, uint16_t* q_out,
                      const kv4_rope& ro, hipStream_t s)
{
    uint16_t *kc = (uint16_t*)c.k + layer * c.g.LS, *vc = (uint16_t*)c.v + layer * c.g.LS;
    const int rows = r.B * r.n, units = (q_out ? n_q : 0) + 2 * c.n_kv, abreast = 2048 / c.head_dim / units;
    auto go = [&](auto kern, int blocks) { kern<<<blocks, 256, 0, s>>>(r, c.g, kc, vc, n_q, c.n_kv, k, v, q, q_out, ro); };
    if (abreast < 2 && c.head_dim == 128) go(k_kv_append<T, 128, true>, rows);
    else if (abreast < 2) go(k_kv_append<T, 64, true>, rows);
    else if (c.head_dim == 128) go(k_kv_append<T, 128, false>, (rows + abreast - 1) / abreast);
    else go(k_kv_append<T, 64, false>, (rows + abreast - 1) / abreast);
}
template void launch_kv_append<float>(const rows_t&, const cache_t&, int, int, kv4_src<float>, kv4_src<float>, kv4_src<float>, uint16_t*,
                                      const kv4_rope&, hipStream_t);
template void launch_kv_append<f32_parts>(const rows_t&, const cache_t&, int, int, kv4_src<f32_parts>, kv4_src<f32_parts>,
                                          kv4_src<f32_parts>, uint16_t*, const kv4_rope&, hipStream_t);
template void launch_kv_append<uint16_t>(const rows_t&, const cache_t&, int, int, kv4_src<uint16_t>, kv4_src<uint16_t>, kv4_src<uint16_t>,
                                         uint16_t*, const kv4_rope&, hipStream_t);

// The plan in the attention itself: each wave's own takes about 3 us, a kernel before it 5 and its launch (8 groups of 8 behind prompts
// of 2048: 40.2 us a call instead of 42.1; one group of 8 behind 512: 14.4 instead of 16.4), unless there are many more
// work-groups than are resident at once.
bool prefix_plans_itself(const px_plan& p, int B) { return B <= PX_WAVE && (long long)B * p.zs <= p.target; }

// Two work-groups a CU are resident.  A slice may have one chunk more than its share of the target (and one more is what the
// share, in floats, may be off).
px_plan prefix_plan(int B, int n, int n_q, int n_kv)
{
    px_plan p = {};
    const int RG = n * (n_q / n_kv);
    p.zs = (RG + PX_ROWS - 1) / PX_ROWS;
    p.sps = p.zs > 1 ? 1 : PX_ROWS / RG < 64 ? PX_ROWS / RG : 64;
    p.target = 512 / n_kv > 1 ? 512 / n_kv : 1;
    p.max_items = p.target + (long long)B * p.zs + 1;
    p.part_rows = (long long)(p.target + 1) * PX_ROWS + (long long)B * RG;
    return p;
}

static size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

size_t prefix_plan_bytes(const px_plan& p, int B, int n_kv, int D)
{
    return up256((size_t)B * sizeof(px_seq)) + up256((size_t)B * sizeof(px_info)) + up256((size_t)p.max_items * sizeof(px_item)) +
           up256((size_t)n_kv * p.part_rows * 8) + up256((size_t)n_kv * p.part_rows * D * 4);
}

void prefix_plan_bind(px_plan& p, void* buf, int B, int n_kv)
{
    char* c = (char*)buf;
    auto take = [&](size_t bytes) {
        char* at = c;
        c += up256(bytes);
        return at;
    };
    p.seq = (px_seq*)take((size_t)B * sizeof(px_seq));
    p.info = (px_info*)take((size_t)B * sizeof(px_info));
    p.item = (px_item*)take((size_t)p.max_items * sizeof(px_item));
    p.ml = (float2*)take((size_t)n_kv * p.part_rows * 8);
    p.o = (float*)c;
}

void launch_prefix_plan(const rows_t& r, const px_groups& g, const px_plan& p, int n_q, int n_kv, hipStream_t s)
{
    const int RG = r.n * (n_q / n_kv);
    if (r.B <= PX_WAVE) k_prefix_plan_wave<<<1, 256, 0, s>>>(r, g, p, RG);
    else k_prefix_plan<<<1, 1024, 0, s>>>(r, g, p, RG);
}

template <int D>
static void prefix_attn_d(const rows_t& r, const px_plan& p, const px_groups& g, const cache_t& c, int n_q, const uint16_t* q, long long q_ld,
                          float cs, void* out, act_t out_t, long long out_ld, hipStream_t s, hipEvent_t ev0, hipEvent_t ev1)
{
    const dim3 grid(c.n_kv, p.max_items);
    const auto kern = p.item ? k_prefix_attn<D, false> : k_prefix_attn<D, true>;
    const uint16_t *kc = (const uint16_t*)c.k, *vc = (const uint16_t*)c.v;
    if (ev0)
        hipExtLaunchKernelGGL(kern, grid, dim3(256), 0, s, ev0, ev1, 0, r, c.g, kc, vc, n_q, c.n_kv, q, q_ld, cs, p, g, out, (int)out_t, out_ld);
    else kern<<<grid, 256, 0, s>>>(r, c.g, kc, vc, n_q, c.n_kv, q, q_ld, cs, p, g, out, (int)out_t, out_ld);
}

void launch_prefix_attention(const rows_t& r, px_plan p, const px_groups& g, const cache_t& c, int layer, int n_q, const uint16_t* q, long long q_ld,
                             float scale, void* out, act_t out_t, long long out_ld, hipStream_t s, hipEvent_t ev0, hipEvent_t ev1)
{
    p.layer = layer;
    const float cs = scale * 1.4426950408889634f;
    if (c.head_dim == 128) prefix_attn_d<128>(r, p, g, c, n_q, q, q_ld, cs, out, out_t, out_ld, s, ev0, ev1);
    else prefix_attn_d<64>(r, p, g, c, n_q, q, q_ld, cs, out, out_t, out_ld, s, ev0, ev1);
}

// Four waves a (row, head) up to so many of them: 4 rows of 16 heads behind 32768 in 256 parts take 25 us a call, with a wave
// 45, 9 x 10 rows of 4 heads behind 8730 24 and 29.  With more of them the parts are fewer: 64 rows of 32 heads in 8 parts 35 us,
// with a wave 33.5 (in 32 parts 72.6 and 75.1).
constexpr int PX_FEW = 512;
void launch_prefix_combine(const rows_t& r, const px_plan& p, int n_q, int n_kv, int D, void* out, act_t out_t, long long out_ld, hipStream_t s)
{
    const long long units = (long long)r.B * r.n * n_q;
    auto go = [&](auto kern, long long blocks) { kern<<<(unsigned)blocks, 256, 0, s>>>(r, p, n_q, n_kv, out, (int)out_t, out_ld); };
    if (units <= PX_FEW) D == 128 ? go(k_prefix_combine<128, 4>, units) : go(k_prefix_combine<64, 4>, units);
    else D == 128 ? go(k_prefix_combine<128, 1>, (units + 3) / 4) : go(k_prefix_combine<64, 1>, (units + 3) / 4);
}
