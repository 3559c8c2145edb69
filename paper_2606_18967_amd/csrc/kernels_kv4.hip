// kernels_kv4.hip -- the paged KV cache in 4 bits: rotary tables, the append
// that rotates, quantizes and stores new rows, the read-back, and the attention
// over it.  Layout and format: sd_kv4_cache in include/sd_api.h.
#include <hip/hip_ext.h>
#include <math.h>

#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// bit of element e in a code word: the elements 2i and 2i + 1 of a word are the
// nibbles 4i bits up in its halves, so one AND makes a pair of fp16 of them
__device__ __forceinline__ constexpr int nib(int e) { return 4 * (e >> 1) + 16 * (e & 1); }

// tile of 32 positions of one KV head (bytes)
constexpr int tile_bytes(int D) { return 32 * D + 256; }

// the page of a slot's positions [lp P, (lp + 1) P), -1 where the block table has
// no valid one
__device__ __forceinline__ int kv4_page(const kv4_geom& g, int slot, int lp)
{
    if (lp < 0 || lp >= g.mpp) return -1;
    const int pg = g.bt[(size_t)slot * g.mpp + lp];
    return pg >= 0 && pg < g.n_pages ? pg : -1;
}

// a first position (kv_len and the like hold anything) kept where sums with row numbers
// stay in 32 bits; past 2^24 either way (the longest cache) no row has a place
__device__ __forceinline__ int kv4_base(long long pos) { return (int)min(max(pos, -(1ll << 25)), 1ll << 25); }

__device__ __forceinline__ void raise(uint32_t* err, int kind)
{
    if (err) flag_error(err, kind);
}

// ------------------------------------------------------------------ rotary table
// table[p][i] = mul (cos p f_i, sin p f_i) in fp64, rounded once.  A work-group
// makes FINE^2 positions of every pair from the sines and cosines of FINE coarse and
// FINE fine angles a pair, cos(a + b) = cos a cos b - sin a sin b: with FINE 16 an
// eighth of the transcendental work, which would bound the kernel, for one more
// rounding in fp64.  What bounds it is a work-group's chain of pow, sincos and two
// barriers, so a short table takes FINE 8, which makes more and shorter groups
// (2048 x 32 pairs 4.6 against 6.4 us; 131072 x 64 22.4 against 18.5, the store
// of 67 MB alone 13).
template <int FINE>
__global__ void __launch_bounds__(512) k_rope_table(sd_rope_cfg c, double lo, double hi, double mul, int n_pos,
                                                    float2* table)
{
    __shared__ double s_f[128];
    __shared__ double2 s_a[FINE * 128], s_b[FINE * 128];
    const int np = c.rot_dim / 2, p0 = blockIdx.x * FINE * FINE;
    for (int i = threadIdx.x; i < np; i += 512) {
        double f = pow(c.theta, -2.0 * i / c.rot_dim);
        if (c.scaling == SD_ROPE_LINEAR) {
            f = f / c.factor;
        } else if (c.scaling == SD_ROPE_LLAMA3) {
            const double t = fmin(fmax((c.orig_ctx * f / 6.283185307179586 - c.low) / (c.high - c.low), 0.0), 1.0);
            f = f * (t + (1.0 - t) / c.factor);
        } else if (c.scaling == SD_ROPE_YARN) {
            const double t = fmin(fmax((i - lo) / fmax(hi - lo, 0.001), 0.0), 1.0);
            f = f * ((1.0 - t) + t / c.factor);
        }
        s_f[i] = f;
    }
    __syncthreads();
    for (int t = threadIdx.x; t < 2 * FINE * np; t += 512) {
        const int k = t / np, i = t - k * np;
        const bool coarse = k < FINE;
        double sn, cs;
        sincos((coarse ? (double)p0 + k * FINE : (double)(k - FINE)) * s_f[i], &sn, &cs);
        if (coarse) s_a[t] = make_double2(cs * mul, sn * mul);
        else s_b[t - FINE * np] = make_double2(cs, sn);
    }
    __syncthreads();
    const int live = min(FINE * FINE, n_pos - p0);
    for (int t = threadIdx.x; t < live * np; t += 512) {
        const int p = t / np, i = t - p * np;
        const double2 a = s_a[p / FINE * np + i], b = s_b[p % FINE * np + i];
        table[(size_t)p0 * np + t] = make_float2((float)(a.x * b.x - a.y * b.y), (float)(a.y * b.x + a.x * b.y));
    }
}

// ------------------------------------------------------------------ append
// A lane's eight dims d0 .. d0 + 7 of a head as they are loaded (words w, values y).
template <typename T> struct oct;
template <> struct oct<float> {
    static constexpr int NW = 8;
    uint32_t w[NW];
    __device__ __forceinline__ void load(const kv4_src<float>& x, size_t i) { put(*(const float4*)(x.x + i), *(const float4*)(x.x + i + 4)); }
    __device__ __forceinline__ void put(float4 a, float4 b)
    {
        const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(v[e]);
    }
    static __device__ __forceinline__ void get(const uint32_t (&w)[NW], float (&y)[8])
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = __uint_as_float(w[e]);
    }
};
template <> struct oct<f32_parts> : oct<float> {
    __device__ __forceinline__ void load(const kv4_src<f32_parts>& x, size_t i)
    {
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
        add_splits2(a, b, x.P, x.S, x.st, i, i + 4);
        put(a, b);
    }
};
template <> struct oct<uint16_t> {
    static constexpr int NW = 4;
    uint32_t w[NW];
    __device__ __forceinline__ void load(const kv4_src<uint16_t>& x, size_t i)
    {
        const u32x4 v = *(const u32x4*)(x.x + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = v[e];
    }
    static __device__ __forceinline__ void get(const uint32_t (&w)[NW], float (&y)[8])
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            y[2 * e] = __uint_as_float(w[e] << 16);
            y[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        }
    }
};

// The dims rotated, the products and their sum in type A, rounded to fp32; t: the
// lane's (cos, sin).  With the half layout a lane's dims turn with those of the lane
// rot/16 further or before.
template <typename A, typename T>
__device__ __forceinline__ void turn(const oct<T>& x, const float2 (&t)[8], int d0, const kv4_rope& ro, float (&y)[8])
{
    x.get(x.w, y);
    if (ro.rot == 0) return;
    if (ro.interleaved) {
        if (d0 >= ro.rot) return;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const A a = y[2 * j], b = y[2 * j + 1], c = t[j].x, s = t[j].y;
            y[2 * j] = (float)(a * c - b * s);
            y[2 * j + 1] = (float)(a * s + b * c);
        }
        return;
    }
    const bool first = d0 < ro.rot / 2;
    const int lane = threadIdx.x & 63, from = d0 >= ro.rot ? lane : first ? lane + ro.rot / 16 : lane - ro.rot / 16;
    uint32_t ow[oct<T>::NW];
    float o[8];
#pragma unroll
    for (int e = 0; e < oct<T>::NW; ++e) ow[e] = __shfl(x.w[e], from, WAVE);
    x.get(ow, o);
    if (d0 >= ro.rot) return;
    const A sg = first ? (A)-1 : (A)1;
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = (float)((A)y[j] * (A)t[j].x + sg * (A)o[j] * (A)t[j].y);
}
// the table's entries for a lane's dims at a position
__device__ __forceinline__ void turns(const kv4_rope& ro, int pos, int d0, float2 (&t)[8])
{
    if (d0 >= ro.rot) return;
    const int h = ro.rot / 2;
    const float4* rp = (const float4*)(ro.table + (size_t)pos * h + (ro.interleaved ? d0 / 2 : d0 < h ? d0 : d0 - h));
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < 2 || !ro.interleaved) {
            const float4 v = rp[j];
            t[2 * j] = make_float2(v.x, v.y);
            t[2 * j + 1] = make_float2(v.z, v.w);
        }
}

// min or max over the D/8 lanes that share a row (neighbours), by lane permutations
// within 16 lanes: i ^ 1, i ^ 2, 7 - i, 15 - i
template <int LPR, typename F>
__device__ __forceinline__ float row_reduce(float v, F f)
{
    auto swap = [&](auto ctrl) {
        return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    v = f(v, swap(std::integral_constant<int, 0xb1>()));
    v = f(v, swap(std::integral_constant<int, 0x4e>()));
    v = f(v, swap(std::integral_constant<int, 0x141>()));
    if (LPR == 16) v = f(v, swap(std::integral_constant<int, 0x140>()));
    return v;
}

// f over the lanes l, l ^ 16, l ^ 32, l ^ 48, in all of them
template <typename F>
__device__ __forceinline__ float across_rows(float v, F f)
{
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// A lane's part of quantizing a row (the group (s, z) of the row's D/8 lanes):
// CODE0 + code of each value, clamp(rint((y - z)/s) + 8, 0, 15).  A sum with
// CODE0 + 8 = 1.5 * 2^23 + 8 rounds to the nearest integer, ties to even.  The
// quotient in fp32 is within 2e-6 of the real one, so it decides unless one is
// within 1e-4 of a half; there (a value in five thousand) fp64 does, whose
// quotient can meet a half only where the real one does.
constexpr uint32_t CODE0 = 0x4b400000u;

template <int LPR>
__device__ __forceinline__ uint32_t quantize8(const float (&y)[8], bool live, uint32_t (&code)[8])
{
    float mn = y[0], mx = y[0], fin = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        mn = fminf(mn, y[e]);
        mx = fmaxf(mx, y[e]);
        fin = __builtin_fmaf(y[e], 0.f, fin);                      // NaN once a value is not finite
    }
    mx = fin == 0.f ? mx : INFINITY;
    mn = row_reduce<LPR>(mn, [](float a, float b) { return fminf(a, b); });
    mx = row_reduce<LPR>(mx, [](float a, float b) { return fmaxf(a, b); });
    const bool bad = mx == INFINITY;
    // (mx - mn) / 15, correctly rounded: the reciprocal's product, and its remainder's
    const double d = (double)mx - (double)mn, r15 = 1.0 / 15.0, q0 = d * r15;
    const uint32_t sb = f32_to_bf16((float)__builtin_fma(__builtin_fma(-15.0, q0, d), r15, q0));
    const float s = __uint_as_float(sb << 16);
    const uint32_t zb = f32_to_bf16((float)__builtin_fma(8.0, (double)s, (double)mn));
    const float z = __uint_as_float(zb << 16), rs = __builtin_amdgcn_rcpf(s);
    float far = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float t = __builtin_amdgcn_fmed3f((y[e] - z) * rs, -8.f, 7.f);
        const float m = t + __uint_as_float(CODE0 + 8);
        far = fmaxf(far, fabsf(t - (m - __uint_as_float(CODE0 + 8))));
        code[e] = __float_as_uint(m);
    }
    // (and steps that are 0, not finite, or without a reciprocal)
    if (__builtin_amdgcn_ballot_w64(live && !(far < 0.4999f && s >= 0x1p-100f && s <= 0x1p100f))) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double q = rint(((double)y[e] - (double)z) / (double)s);
            code[e] = CODE0 + (s > 0.f && !bad ? (uint32_t)((int)fmin(fmax(q, -8.0), 7.0) + 8) : 8u);
        }
    }
    return bad ? 0x7fc07fc0u : sb | zb << 16;
}

// One wave takes the new rows among 8 consecutive positions of one KV head's K or
// V (the words of V hold 8 positions, so a word has one writer), D/8 lanes a row;
// further waves rotate the queries, D/8 lanes a head, q_passes times 512/D heads of
// a row each.  K is rotated in fp64 so that its codes are those of the exact rotation (a
// value next to a border moves by a whole step otherwise); its products are few
// against the row's bytes.
// Few rows are bound by the chain of loads length, page, row, and a V word's other
// nibbles: a row of 32 / 8 heads of 128 takes 4.3 us, 64 x 5 rows of 40 / 8 7.5 (both
// halves of a group's words in scattered pages).  Many are bound by memory: 16 x 1536 rows
// of 32 / 8 heads 112 us (4.7 TB/s).  Rows that are absent cost their waves' start and
// leave: half of those rows 66 us (4.0 TB/s), as many in a call without absent ones 61;
// 10722 of them in ragged lengths 60.
// A wave takes one KV head, or where there are more than KV4_APPEND_WAVES of them its
// group's heads one after the other, the next one's loads under way, and positions and table
// entries once (16 x 1536 rows, 2048 and 4096 waves at least 115 us, 8192 120, a head a wave
// always 143; 16 x 100 rows 1024 14.1, 4096 13.1).  Query passes a wave: 1, 2, 4 of
// them 158, 129, 115 us; with few rows, as split-K partials have, 2 (64 x 5: 6.4, 4: 6.7).
template <typename T>
constexpr int q_passes() { return std::is_same<T, f32_parts>::value ? 2 : 4; }
constexpr int KV4_APPEND_WAVES = 4096;

template <typename T, int D>
__global__ void __launch_bounds__(256) k_kv4_append(rows_t r, kv4_geom g, int n_q, int n_kv, kv4_src<T> xk, kv4_src<T> xv,
                                                    kv4_src<T> xq, uint16_t* q_out, kv4_rope ro, int ngr, int hpw, int kv_waves)
{
    constexpr int LPR = D / 8, RPW = WAVE / LPR, NP = 8 / RPW;     // lanes a row, rows a pass, passes of a group
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const int lw = lane % LPR, lt = lane / LPR, d0 = 8 * lw;
    if (wave >= kv_waves) {                                        // queries: QH heads of one row
        if (!q_out) return;                                        // the last work-group's waves past K and V
        constexpr int QPASS = q_passes<T>(), QH = QPASS * RPW;
        const int qw = (n_q + QH - 1) / QH, unit = wave - kv_waves, idx = unit / qw, hb = (unit - idx * qw) * QH, h0 = hb + lt;
        const int b = idx / r.n, i = idx - b * r.n;
        if (b >= r.B || (r.lim && i >= r.lim[b])) return;
        const size_t row = r.row0 ? r.row0[b] + i : idx;
        const int slot = r.slots[b];
        int pos = -1;
        if (slot >= 0 && slot < r.max_slots) pos = kv4_base((long long)r.kv_len[slot] + r.off) + i;
        const bool ok = pos >= 0 && pos < r.max_ctx && (ro.rot == 0 || pos < ro.len);
        float2 tr[8] = {};
        oct<T> x[QPASS] = {};
        if (ok) {
#pragma unroll
            for (int ps = 0; ps < QPASS; ++ps)                     // past the last head: it again, not stored
                if (hb + ps * RPW < n_q) x[ps].load(xq, row * xq.ld + (size_t)min(h0 + ps * RPW, n_q - 1) * D + d0);
            turns(ro, pos, d0, tr);
        }
#pragma unroll
        for (int ps = 0; ps < QPASS; ++ps) {
            if (hb + ps * RPW >= n_q) break;
            float y[8];
            turn<float>(x[ps], tr, d0, ro, y);
            if (h0 + ps * RPW < n_q)
                *(u32x4*)(q_out + (row * n_q + h0 + ps * RPW) * D + d0) =
                    (u32x4){pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])};
        }
        return;
    }
    // (sequence, group, hpw KV heads, K or V), the heads of one group side by side
    const int hw = (n_kv + hpw - 1) / hpw;
    const int u = wave % (2 * hw), bg = wave / (2 * hw), b = bg / ngr, gr = bg - b * ngr;
    const bool is_v = u >= hw;
    const int h0 = (is_v ? u - hw : u) * hpw, h1 = min(h0 + hpw, n_kv);
    const int nl = r.lim ? r.lim[b] : r.n, nlive = min(max(nl, 0), r.n);
    const int slot = r.slots[b];
    const bool first = gr == 0 && u == 0 && lane == 0;
    if (first && nl != nlive) raise(r.err, ERR_LEN);
    if (slot < 0 || slot >= r.max_slots) {
        if (first && nlive > 0) raise(r.err, ERR_SLOT);
        return;
    }
    const int base = kv4_base((long long)r.kv_len[slot] + r.off);
    const int stop = ro.rot ? min(r.max_ctx, ro.len) : r.max_ctx;  // first position without a table row or a place
    if (first && nlive > 0 && (base < 0 || base > stop - nlive)) raise(r.err, ERR_CTX);
    // the group's positions [pg0, pg0 + 8), the rows' [lo, hi)
    const int pg0 = ((base < 0 ? 0 : base) & ~7) + 8 * gr, lo = max(max(base, 0), pg0);
    const int hi = min(pg0 + 8, (int)min((long long)stop, (long long)base + nlive));
    if (lo >= hi) return;
    const int page = kv4_page(g, slot, pg0 / g.P);                 // a page holds whole groups
    if (page < 0) {
        if (u == 0 && lane == 0) raise(r.err, ERR_PAGE);
        return;
    }
    const int in = pg0 % g.P, r32 = in & 31;
    uint8_t* tile = g.pages + page * g.PS + h0 * g.HS + (size_t)(in >> 5) * tile_bytes(D);
    const size_t row0 = r.row0 ? r.row0[b] : (size_t)b * r.n;
    auto store = [&](auto vtag) {
        constexpr bool V = decltype(vtag)::value;
        const kv4_src<T>& src = V ? xv : xk;
        const kv4_rope rk = V ? kv4_rope{nullptr, 0, 0, 0} : ro;
        oct<T> next[NP] = {};
        float2 tr[NP][8] = {};
        auto fetch = [&](int h) {
#pragma unroll
            for (int ps = 0; ps < NP; ++ps) {
                const int pos = pg0 + ps * RPW + lt;
                if (pos >= lo && pos < hi) next[ps].load(src, (row0 + (pos - base)) * src.ld + (size_t)h * D + d0);
            }
        };
        fetch(h0);
#pragma unroll
        for (int ps = 0; ps < NP; ++ps) {
            const int pos = pg0 + ps * RPW + lt;
            if (pos >= lo && pos < hi) turns(rk, pos, d0, tr[ps]);
        }
        uint32_t mask = 0;                                         // the new rows' nibbles of a V word
#pragma unroll
        for (int t = 0; t < 8; ++t)
            if (pg0 + t >= lo && pg0 + t < hi) mask |= 0xfu << nib(t);
        for (int h = h0; h < h1; ++h, tile += g.HS) {
            oct<T> now[NP];
#pragma unroll
            for (int ps = 0; ps < NP; ++ps) now[ps] = next[ps];
            if (h + 1 < h1) fetch(h + 1);
            uint32_t vw[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int ps = 0; ps < NP; ++ps) {
                const int t = ps * RPW + lt, pos = pg0 + t;
                const bool live = pos >= lo && pos < hi;
                float y[8];
                uint32_t code[8];
                turn<double>(now[ps], tr[ps], d0, rk, y);
                const uint32_t par = quantize8<LPR>(y, live, code);
                if (V) {
                    const int sh = nib(t);
                    const uint32_t take = live ? 15u : 0u;
#pragma unroll
                    for (int e = 0; e < 8; ++e) vw[e] |= (code[e] & take) << sh;
                } else if (live) {
                    uint32_t w = 0, zero = 0;                      // sum (CODE0 + code) 2^nib, less that of CODE0
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        w += code[e] << nib(e);
                        zero += CODE0 << nib(e);
                    }
                    *(uint32_t*)(tile + (r32 + t) * (D / 2) + 4 * lw) = w - zero;
                }
                if (live && lw == 0) *(uint32_t*)(tile + 32 * D + (V ? 128 : 0) + 4 * (r32 + t)) = par;
            }
            if (!V) continue;
            // a word's nibbles lie in the lanes lw of every lt: each exchange leaves a lane
            // half of the words, until lane (lt, lw) has its 8 / RPW of them
            constexpr int WPL = 8 / RPW;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const auto x = __builtin_amdgcn_permlane32_swap(vw[e], vw[e + 4], false, false);
                vw[e] = x[0] | x[1];
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const auto x = __builtin_amdgcn_permlane16_swap(vw[e], vw[e + 2], false, false);
                vw[e] = x[0] | x[1];
            }
            int w0 = (lane & 32 ? 4 : 0) + (lane & 16 ? 2 : 0);
            if (WPL == 1) {
                const uint32_t got = __builtin_amdgcn_mov_dpp(lane & 8 ? vw[0] : vw[1], 0x128, 0xf, 0xf, true);   // lane ^ 8
                vw[0] = (lane & 8 ? vw[1] : vw[0]) | got;
                w0 += lane & 8 ? 1 : 0;
            }
            uint32_t* dst = (uint32_t*)(tile + 16 * D) + (r32 >> 3) * D + d0 + w0;
#pragma unroll
            for (int e = 0; e < WPL; ++e) dst[e] = mask == 0xffffffffu ? vw[e] : (dst[e] & ~mask) | vw[e];
        }
    };
    if (is_v) store(std::true_type());
    else store(std::false_type());
}

// ------------------------------------------------------------------ read
// A thread takes 8 dims of K or V of the rows among 8 consecutive positions, so a V word
// is read once (12288 rows of 8 heads of 128: 19 us, 3.3 TB/s; 24576 33 us, 3.8; one row
// 3.0).  What bounds it is its many narrow loads: K words of 4 bytes a lane, and the eight
// rows' groups in every lane of them.
template <int D>
__global__ void __launch_bounds__(256) k_kv4_read(rows_t r, kv4_geom g, int n_kv, uint16_t* k_out, uint16_t* v_out,
                                                  const int32_t* start, int ngr, long long total)
{
    constexpr int LPR = D / 8;
    const long long t0 = (long long)blockIdx.x * 256 + threadIdx.x;
    if (t0 >= total) return;
    const int lw = (int)(t0 % LPR);
    const long long un = t0 / LPR;
    const int u = (int)(un % (2 * n_kv)), bg = (int)(un / (2 * n_kv)), b = bg / ngr, gr = bg - b * ngr;
    const bool is_v = u >= n_kv;
    const int h = is_v ? u - n_kv : u;
    const int nl = r.lim ? r.lim[b] : r.n, nlive = min(max(nl, 0), r.n);
    const int slot = r.slots[b], base = start[b];
    const bool first = gr == 0 && u == 0 && lw == 0;
    if (first) {
        if (nl != nlive) raise(r.err, ERR_LEN);
        if (nlive > 0 && (slot < 0 || slot >= r.max_slots)) raise(r.err, ERR_SLOT);
        if (nlive > 0 && (base < 0 || base > r.max_ctx - nlive)) raise(r.err, ERR_CTX);
    }
    // rows i of the group gr: positions 8 (base / 8 + gr) + t (base rounded down, also below 0)
    const long long pg0 = (long long)(base & ~7) + 8 * gr;
    int page = -1;
    if (slot >= 0 && slot < r.max_slots && pg0 >= 0 && pg0 < r.max_ctx) {
        page = kv4_page(g, slot, (int)(pg0 / g.P));
        if (page < 0 && u == 0 && lw == 0 && pg0 < (long long)base + nlive) raise(r.err, ERR_PAGE);
    }
    uint32_t w[8], par[8];
    if (page >= 0) {
        const int in = (int)(pg0 % g.P), r32 = in & 31;
        const uint8_t* tile = g.pages + page * g.PS + h * g.HS + (size_t)(in >> 5) * tile_bytes(D);
        const uint32_t* src = is_v ? (const uint32_t*)(tile + 16 * D) + (r32 >> 3) * D + 8 * lw
                                   : (const uint32_t*)(tile + r32 * (D / 2)) + lw;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            w[e] = src[is_v ? e : e * (D / 8)];
            par[e] = ((const uint32_t*)(tile + 32 * D + (is_v ? 128 : 0)))[r32 + e];
        }
    }
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        const long long i = pg0 + t - base;
        if (i < 0 || i >= nlive) continue;
        float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (page >= 0 && pg0 + t < r.max_ctx) {
            const float s = __uint_as_float(par[t] << 16), z = __uint_as_float(par[t] & 0xffff0000u);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t c = (is_v ? w[e] >> nib(t) : w[t] >> nib(e)) & 15u;
                y[e] = __builtin_fmaf(s, (float)((int)c - 8), z);
            }
        }
        uint16_t* o = (is_v ? v_out : k_out) + (((size_t)b * r.n + (size_t)i) * n_kv + h) * D + 8 * lw;
        *(u32x4*)o = (u32x4){pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]),
                             pack_bf16x2(y[6], y[7])};
    }
}

// ------------------------------------------------------------------ attention
__device__ __forceinline__ void kv4_store4(void* out, int out_t, size_t i, float4 v)
{
    if (out_t == ACT_F16) {
        const half2v a = {(_Float16)v.x, (_Float16)v.y}, b = {(_Float16)v.z, (_Float16)v.w};
        *(uint2*)((_Float16*)out + i) = make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
    } else {
        *(uint2*)((uint16_t*)out + i) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    }
}

// partial result (ref, l, o[D]) of query row qrow (of QR a KV head) of an item
__device__ __forceinline__ size_t part_at(int item, int n_kv, int kvh, int QR, int qrow, int D)
{
    return (((size_t)item * n_kv + kvh) * QR + qrow) * (D + 4);
}

// The item of a work-group without a plan in memory (plan.item NULL), as
// launch_attention_plan would make it: the sequence itself where every one is an
// item in order, else, of up to 64 sequences (a lane each), the cut whose chunk
// length is the shortest of 64 candidates that makes at most `target` items.  A
// wave needs a microsecond for it, where a launch before the attention and the
// way through memory take four.  nch also tells the combine (plan.seq).
__device__ att_item own_item(const rows_t& r, const att_plan& pl, int item)
{
    const int lane = threadIdx.x & 63, b = pl.whole ? item : lane;
    att_item it = {0, -1, 0, 0, 0, 0, 0, 0};
    if (b < r.B) {
        it.row0 = b * r.n;
        it.slot = r.slots[b];
        const int nl = r.lim ? r.lim[b] : r.n;
        it.nlive = min(max(nl, 0), r.n);
        if (nl != it.nlive) raise(r.err, ERR_LEN);
        it.nch = 1;
        if (it.slot >= 0 && it.slot < r.max_slots) {
            it.basepos = r.kv_len[it.slot];
            it.ctx = (int)max(0ll, min((long long)it.basepos + it.nlive, (long long)r.max_ctx));
        }
        it.p1 = it.ctx;
    }
    if (pl.whole) return it;
    int sum = it.ctx, top = it.ctx;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        sum += __shfl_xor(sum, o, WAVE);
        top = max(top, __shfl_xor(top, o, WAVE));
    }
    const plan_cut c = plan_candidates(sum, top, pl);
    const int ck = c.at(lane);
    const float rc = 1.f / (float)ck;
    // chunks of ctx positions, at most some hundred: one correction makes the quotient exact
    auto chunks = [](int ctx, int ch, float rc) {
        int q = (int)((float)ctx * rc);
        q += q * ch < ctx;
        return max(q, 1);
    };
    int cnt = 0;
    for (int s = 0; s < r.B; ++s) cnt += chunks(__builtin_amdgcn_readlane(it.ctx, s), ck, rc);
    const uint64_t fits = __builtin_amdgcn_ballot_w64(cnt <= min(pl.target, pl.max_items));
    const int ch = c.at(fits ? (int)__builtin_ctzll(fits) : 63);
    const int nch = b < r.B ? chunks(it.ctx, ch, 1.f / (float)ch) : 0;
    int upto = nch;                                                // inclusive sum over the wave
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(upto, o, WAVE);
        if (lane >= o) upto += v;
    }
    const uint64_t mine = __builtin_amdgcn_ballot_w64(upto > item);
    att_item none = {0, -1, 0, 0, 0, 0, 0, 0};
    if (!mine) return none;                                        // past the last item
    const int s = __builtin_ctzll(mine);
    it.nch = nch;
    auto from = [&](int v) { return __builtin_amdgcn_readlane(v, s); };
    const int first = from(upto) - from(nch);
    it = att_item{from(it.row0), from(it.slot), from(it.basepos), from(it.ctx), 0, 0, from(it.nch), from(it.nlive)};
    const int len = ((it.ctx + it.nch - 1) / it.nch + PLAN_UNIT - 1) / PLAN_UNIT * PLAN_UNIT;
    it.p0 = min((item - first) * len, it.ctx);
    it.p1 = min(it.p0 + len, it.ctx);
    if (item == first && threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.z == 0) pl.seq[s] = make_int2(first, it.nch);
    return it;
}

// Work-group (item, KV head, slice of 16 MQ query rows) covers the positions
// [p0, p1) of its item (att_plan); its four waves take the tiles of 32 positions
// in turn.  With q the query, c the codes of a position and (s, z) its group,
//   score = s (q . c - 8 sum(q)) + z sum(q),   out = sum (P s) (c - 8) + sum P z,
// so the products run on the codes themselves.  A nibble under a mask is an fp16
// number as it stands: c 2^-24 in bits 0..3 (denormal, which the matrix cores
// take), c 2^-20 in bits 4..7; a word's eight codes are four ANDs and a shift,
// and the other operand's elements 2, 3, 6 and 7 carry the factor 1/16.
//   S^T = K Q^T with v_mfma_f32_16x16x32_f16, the queries scaled by a power of
// two (see the query fragments).  Row j of tile half pt is position
// 8 (j/4) + 4 pt + j%4, so that a lane's eight scores are the positions
// 8 (lane/16) + 0..7 of query row lane % 16: the B operand of O^T += V^T P^T, whose
// A operand is one word of V codes a lane (8 positions of one dim).  P s goes in
// as fp16, 2^-11 of each where the output's own rounding is 2^-8 (the error against 64
// bits of the outputs is 1.66e-3 with P in 32 bits, 1.68e-3 so, at 131071 positions
// 1.71e-3), and one more product with codes of 8 sums what the centre takes off again.
// Online softmax in base 2.  A row's reference ref bounds the products' operand:
// P s = exp2(score - ref) s <= 2^15; it moves, with all sums, only where a tile
// would exceed that, to where the tile's largest P s is 2^7, so small terms are
// off by 2^-28 of a row's largest (of elements over 16; the others by 2^-32).  P itself
// stays below 2^75 where s is smaller than 2^-60.  Sums and statistics in fp32.
//   What bounds it: single rows the cache's bytes (64 sequences of 32 or 40 / 8 heads of 128
// at 2048, 8192 and 32768 positions 28, 94 and 342 us: 5.1, 6.1 and 6.7 TB/s; a launch and
// the first tiles' way take 5); one short sequence its chain of launch, plan, page,
// tile (2048 positions 7.7 us, the combine 4); 64 x 5 verify rows at 8192 positions
// bytes and vector units alike (105 to 116 us on different boxes, 5 to 5.5 TB/s); a
// prefill the vector units: 46 cycles a score of 64 lanes in the softmax, 5 instructions
// a code word, 17 products of 16 cycles a 16-row tile (8 x 512 rows at 4096 positions
// 306 us, 840 TFLOP/s).
constexpr float KV4_REF0 = -3.4028235e38f;     // the reference of a row that has seen no position: below every score

// 64 lanes x 16 (or 4) bytes at base + off straight into LDS, in lane order from byte
// `lds` on; non-temporal.  The compiler's wait counts do not see them.
__device__ __forceinline__ void tile_dma16(const void* base, uint32_t off, uint32_t lds)
{
    asm volatile("global_load_lds_dwordx4 %0, %1 nt" : : "v"(off), "s"(base), "{m0}"(lds) : "memory");
}
__device__ __forceinline__ void tile_dma4(const void* base, uint32_t off, uint32_t lds)
{
    asm volatile("global_load_lds_dword %0, %1 nt" : : "v"(off), "s"(base), "{m0}"(lds) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_tiles()
{
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

//
// ROWS, for many query rows: the four waves take 16 MQ rows each instead, and every
// tile, which they fetch together into one ring (a quarter of its codes each; the
// groups each for itself): the cache is read once for 64 MQ rows and nothing is
// merged.
template <int D, int MQ, bool ROWS>
__global__ void __launch_bounds__(256, 2) k_kv4_attn(rows_t r, kv4_geom g, int n_q, int n_kv,
                                                                   const uint16_t* q, long long q_ld, float cs,
                                                                   float* part, att_plan plan, void* out, int out_t,
                                                                   long long out_ld)
{
    constexpr int KW = D / 32;       // code words of a lane's part of a K row: k-steps of S
    constexpr int NBD = D / 16;      // 16-row blocks of O^T, code words of a lane's V
    constexpr int LDO = D + 4;       // LDS row stride of the merge
    constexpr int TB = tile_bytes(D), PIECES = ROWS ? 2 : D / 32 + 1;   // a wave's loads of a tile
    constexpr int RING = ROWS ? 3 : 2;                             // tiles in LDS or on the way (one more: the same times)
    constexpr int SLOT = ROWS ? 32 * D + 4 * 256 : TB;             // a ring's place: the tile, or its codes and four times its groups
    constexpr int RINGS = ROWS ? RING * SLOT : 4 * RING * SLOT, MERGE = ROWS ? 0 : 4 * 16 * LDO * 4;
    constexpr int STEP = ROWS ? 32 : 128;                          // positions between a wave's tiles
    __shared__ __attribute__((aligned(1024))) uint8_t s_buf[RINGS > MERGE ? RINGS : MERGE];   // the rings, then the merge
    __shared__ float2 s_par[4 * 64];
    __shared__ float s_ml[4][2][16];
    __shared__ float s_back[4][MQ][16];                            // rows apart: what gives a row's power of two back

    const int item = blockIdx.y, kvh = blockIdx.x, zsl = gridDim.z - 1 - blockIdx.z;   // the last rows, which see most, first
    const att_item it = plan.item ? plan.item[item] : own_item(r, plan, item);
    if (it.nch == 0) return;
    const int row0 = __builtin_amdgcn_readfirstlane(it.row0), slot = __builtin_amdgcn_readfirstlane(it.slot);
    const int basepos = kv4_base(__builtin_amdgcn_readfirstlane(it.basepos));
    const int p0 = __builtin_amdgcn_readfirstlane(it.p0), p1 = __builtin_amdgcn_readfirstlane(it.p1);
    const int nlive = __builtin_amdgcn_readfirstlane(it.nlive);
    // the sequence's query rows, the G heads of a position side by side (QR of them; a stored item has room for G n)
    const int G = n_q / n_kv, QR = G * nlive;
    constexpr int SROWS = ROWS ? 64 * MQ : 16 * MQ;                // the slice's rows, and the wave's
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int qslice = zsl * SROWS, qbase = ROWS ? qslice + 16 * MQ * w : qslice;
    if (qslice >= QR) return;                                      // a slice past them
    if (p0 == 0 && zsl == 0 && kvh == 0 && threadIdx.x == 0) {
        if (slot < 0 || slot >= r.max_slots) raise(r.err, ERR_SLOT);
        else if (basepos < 0 || basepos > r.max_ctx - nlive) raise(r.err, ERR_CTX);
    }
    const int cq = lane >> 4, lr = lane & 15;
    // past the last position that a live row of rows [q0, q0 + rows) sees
    auto seen_to = [&](int q0, int rows) {
        const int last = min(q0 + rows, QR) - 1;
        return last < q0 ? p0 : min(p1, basepos + last / G + 1);
    };
    const int pe = seen_to(qbase, 16 * MQ), pslice = seen_to(qslice, SROWS);
    // up to where all of the wave's rows see everything
    const int all = basepos + qbase / G;

    // tile i of the wave is at positions wq0 + STEP i; nt tiles are fetched, of which it uses `own`
    const int wq0 = ROWS ? p0 : p0 + 32 * w;
    const bool usable = slot >= 0 && slot < r.max_slots;           // else p0 == p1 == 0: no tile
    const int nt = usable ? max(pslice - wq0 + STEP - 1, 0) / STEP : 0, own = ROWS ? min(nt, max(pe - wq0 + STEP - 1, 0) / STEP) : nt;
    // Those that every row sees as a whole come first, each item's from another one on:
    // sequences of a size whose pages lie in order read the same memory channels at a
    // time otherwise (64 at 8192 positions in pages of 64, of 256: 102 and 112 us, 94 and
    // 96 so; pages in random order 98 and 97).
    // (rows past max_ctx see nothing: with one of them every tile is masked)
    const int whole = basepos > r.max_ctx - nlive ? 0 : min(own, max(0, (min(pe, all + 1) - wq0 + STEP - 32) / STEP));
    const int from = ROWS || whole == 0 ? 0 : item * 13 % whole;
    auto place = [&](int i) { return ROWS || i >= whole ? i : i + from < whole ? i + from : i + from - whole; };
    const uint8_t* slots_at = s_buf + (ROWS ? 0 : w * (RING * SLOT));
    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)slots_at;
    const uint8_t* head = g.pages + kvh * g.HS;
    // a lane's pieces of a tile: K row 8 (lr/4) + 4 pt + lr%4, words (D/32) cq + 0..; V group cq, words NBD lr + 0..
    constexpr int NSRC = D / 32 + 1;
    uint32_t src[NSRC];
    if constexpr (D == 128) {
        src[0] = (8 * (lr >> 2) + (lr & 3)) * 64 + cq * 16;
        src[1] = src[0] + 256;
        src[2] = 2048 + cq * 512 + lr * 32;
        src[3] = src[2] + 16;
    } else {
        src[0] = 16 * lane;
        src[1] = 1024 + 16 * lane;
    }
    src[NSRC - 1] = 32 * D + 4 * lane;                             // the groups: 64 lanes x 4 bytes
    if constexpr (ROWS) {                                          // the wave's quarter of the codes (of 64 dims 32 lanes of it)
        if constexpr (D == 128) src[0] = w == 0 ? src[0] : w == 1 ? src[1] : w == 2 ? src[2] : src[3];
        else src[0] = 512 * w + 16 * lane;
    }
    // the pages of the steps [kw, kw + 128), lane l holding those of kw + l and
    // kw + 64 + l (-1: missing): one table load in 128 tiles
    int pgw[2] = {-1, -1}, kw = -(1 << 20);
    uint32_t there = 0;                                            // bit i % 32: step i's tile has a page
    auto issue = [&](int i, int at) {
        if (i < kw || i >= kw + 128) {
            kw = i;
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                const int bj = wq0 + place(i + 64 * hf + lane) * STEP;
                pgw[hf] = bj < pslice ? kv4_page(g, slot, bj / g.P) : -1;
                if (pgw[hf] < 0 && bj < pslice && r.err) ((volatile __attribute__((address_space(1))) uint32_t*)r.err)[ERR_PAGE] = 1u;
            }
        }
        const int j = i - kw, blk = wq0 + STEP * place(i), in = __builtin_amdgcn_readfirstlane(blk % g.P);
        const int pa = __builtin_amdgcn_readlane(pgw[0], j & 63), pb = __builtin_amdgcn_readlane(pgw[1], j & 63);
        const int pg = j < 64 ? pa : pb;
        there = (there & ~(1u << (i & 31))) | (uint32_t)(pg >= 0) << (i & 31);
        // no page: the first tile of the pool is fetched and not used, so that every tile counts alike
        const uint8_t* t = head + (pg < 0 ? 0 : pg * g.PS + (in >> 5) * (long long)TB);
        const uint32_t to = ring + at * SLOT;
        if constexpr (ROWS) {
            if (D == 128 || lane < 32) tile_dma16(t, src[0], to + 8 * D * w);
            tile_dma4(t, src[NSRC - 1], to + 32 * D + 256 * w);
        } else {
#pragma unroll
            for (int k = 0; k < NSRC - 1; ++k) tile_dma16(t, src[k], to + 1024 * k);
            tile_dma4(t, src[NSRC - 1], to + 32 * D);
        }
    };
    // (the barrier that opens a tile of a common ring frees the one before)
    constexpr int AHEAD = ROWS ? RING - 1 : RING;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
        if (u < nt) issue(u, u);

    // query fragments: row lr's dims (D/4) cq + 8 ks + 0..7 times the power of two that puts the largest
    // below 2^14, elements 2, 3, 6, 7 over 16; the row's sum in the products' unit (2^-24); and the factor from that
    // unit to a score in base 2.  Rows of a size share one power of two, which the tiles' groups then carry: a bf16
    // value keeps all its bits down to 2^-26 of the slice's largest (elements over 16; the others to 2^-30) and is off by
    // 2^-34 of it below that, 2^-25 of the largest of a row whose exponent is 8 less.  Where one is smaller, or infinite,
    // or the common factor could leave fp32, the rows are `apart`: each has its own power of two, which the products give
    // back on the path that moves references, and an infinite or NaN query stays in its row.  That path takes longer (us,
    // with one head's queries 2^10 times the others': 64 rows at 8192 positions of 40 / 8 heads 100 instead of 92, 64 x 5
    // 178 and 108, 8 x 512 at 4096 642 and 314).
    half8 qf[MQ][KW];
    float qsum[MQ], unit;
    uint64_t apart;                                                // 0 or a ballot
    int lim[MQ];
    floatx4 mid8[MQ];                                              // what the centre 8 takes off a score's products
    {
        u32x4 v[MQ][KW];
        float top[MQ], most = 0.f;
        auto larger = [](float a, float b) { return fmaxf(a, b); };
#pragma unroll
        for (int mt = 0; mt < MQ; ++mt) {
            const int qrow = qbase + 16 * mt + lr, i = qrow / G, h = qrow - i * G, pos = basepos + i;
            const bool live = qrow < QR && pos >= 0 && pos < r.max_ctx;
            lim[mt] = live ? pos : -1;
            const uint16_t* qp = q + (size_t)(row0 + (live ? i : 0)) * q_ld + (size_t)(kvh * G + (live ? h : 0)) * D + (D / 4) * cq;
            top[mt] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KW; ++ks) {
                v[mt][ks] = live ? *(const u32x4*)(qp + 8 * ks) : (u32x4){0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    top[mt] = fmaxf(top[mt], fmaxf(fabsf(__uint_as_float(v[mt][ks][e] << 16)), fabsf(__uint_as_float(v[mt][ks][e] & 0xffff0000u))));
            }
            top[mt] = across_rows(top[mt], larger);
            most = fmaxf(most, top[mt]);
        }
        auto exponent = [](float x) { return (int)(__float_as_uint(x) >> 23); };
        const int em = exponent(row_reduce<16>(most, larger));
        bool far = em > 187;                                       // 2^61
#pragma unroll
        for (int mt = 0; mt < MQ; ++mt) far |= top[mt] > 0.f && exponent(top[mt]) < em - 8;
        apart = __builtin_amdgcn_ballot_w64(far);
        auto shift_of = [](int e) { return min(267 - e, 253); };   // biased, of the power of two for a largest of exponent e
        auto back_of = [&](int e) { return __uint_as_float((uint32_t)(254 - shift_of(e)) << 23); };
        unit = apart ? cs : cs * back_of(em) * 16777216.f;
#pragma unroll
        for (int mt = 0; mt < MQ; ++mt) {
            const int er = apart ? exponent(top[mt]) : em;
            const float up = __uint_as_float((uint32_t)shift_of(er) << 23);
            const float back = back_of(er);
            s_back[w][mt][lr] = back;
            float sum = 0.f;
#pragma unroll
            for (int ks = 0; ks < KW; ++ks)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float a = __uint_as_float(v[mt][ks][e] << 16) * up, b = __uint_as_float(v[mt][ks][e] & 0xffff0000u) * up;
                    sum += a + b;
                    const float f = e & 1 ? 0.0625f : 1.f;
                    qf[mt][ks][2 * e] = (_Float16)(a * f);
                    qf[mt][ks][2 * e + 1] = (_Float16)(b * f);
                }
            sum = across_rows(sum, [](float a, float b) { return a + b; });
            const float in_unit = sum * 5.9604644775390625e-08f;   // 2^-24
            mid8[mt] = (floatx4){-8.f * in_unit, -8.f * in_unit, -8.f * in_unit, -8.f * in_unit};
            qsum[mt] = apart ? sum * back : in_unit;
        }
    }
    // a tile's groups in fp32, a lane a group: (s, z) of a key in score units, (s, z) of a
    // value with the operand's 1/16
    float2* par = (float2*)(s_par + 64 * w);
    const float par_s = lane < 32 ? unit : lane & 2 ? 0.0625f : 1.f, par_z = lane < 32 ? unit : 1.f;

    float limit = apart ? -1.f : 32768.f;                          // of P s; -1: every tile takes the path that moves references
    float ref[MQ], lsum[MQ], zsum[MQ];
    floatx4 o[MQ][NBD], oc[MQ];
#pragma unroll
    for (int mt = 0; mt < MQ; ++mt) {
        ref[mt] = KV4_REF0;
        lsum[mt] = zsum[mt] = 0.f;
        oc[mt] = (floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int nb = 0; nb < NBD; ++nb) o[mt][nb] = (floatx4){0.f, 0.f, 0.f, 0.f};
    }

    // a word's codes in fp16 (see above)
    auto codes = [](uint32_t x) {
        const uint32_t y = x >> 8;
        return __builtin_bit_cast(half8, (u32x4){x & 0x000f000fu, x & 0x00f000f0u, y & 0x000f000fu, y & 0x00f000f0u});
    };
    auto block = [&](int blk, const uint8_t* t, auto masked) {
        constexpr bool MASKED = decltype(masked)::value;
        alignas(16) uint32_t kc[2][KW], vc[NBD];
        const uint32_t raw = *(const uint32_t*)(t + 32 * D + (ROWS ? 256 * w : 0) + 4 * lane);
        if constexpr (D == 128) {
            *(u32x4*)kc[0] = *(const u32x4*)(t + 16 * lane);
            *(u32x4*)kc[1] = *(const u32x4*)(t + 1024 + 16 * lane);
        } else {
            const uint8_t* kr = t + (8 * (lr >> 2) + (lr & 3)) * 32 + cq * 8;
            *(u32x2*)kc[0] = *(const u32x2*)kr;
            *(u32x2*)kc[1] = *(const u32x2*)(kr + 128);
        }
        const float step = __uint_as_float(raw << 16);
        par[lane] = make_float2(step * par_s, __uint_as_float(raw & 0xffff0000u) * par_z);
        // (values that are all alike have s = 0: P needs a bound of its own)
        const bool tiny = __builtin_amdgcn_ballot_w64(lane >= 32 && !(step >= 0x1p-60f)) != 0;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        floatx4 st[MQ][2];
        __builtin_amdgcn_sched_barrier(0);                         // the products start together (64 x 5 rows: 112 -> 108 us)
#pragma unroll
        for (int pt = 0; pt < 2; ++pt)
#pragma unroll
            for (int k = 0; k < KW; ++k) {
                const half8 kf = codes(kc[pt][k]);
#pragma unroll
                for (int mt = 0; mt < MQ; ++mt)
                    st[mt][pt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[mt][k], k ? st[mt][pt] : mid8[mt], 0, 0, 0);
            }
        float ks[8], kz[8], vs[8], vz[8];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const float4 a = *(const float4*)(par + 8 * cq + e), b = *(const float4*)(par + 32 + 8 * cq + e);
            ks[e] = a.x, kz[e] = a.y, ks[e + 1] = a.z, kz[e + 1] = a.w;
            vs[e] = b.x, vz[e] = b.y, vs[e + 1] = b.z, vz[e + 1] = b.w;
        }
        // The vector units bound a tile (some 1250 cycles of them beside 550 of products, D =
        // 128, MQ = 2), so a wave in its softmax goes before one that waits on its products.
        // With and without, us: 64 x 5 rows at 8192 positions of 40 / 8 heads 108 / 115, 8 x 512
        // at 4096 of 32 / 8 312 / 335, single rows alike.
        __builtin_amdgcn_s_setprio(1);
        half8 pf[MQ];
#pragma unroll
        for (int mt = 0; mt < MQ; ++mt) {
            float p[8], pv[8];
            bool seen[8];
            const int last = min(pe - 1, lim[mt]);
#pragma unroll
            for (int e = 0; e < 8; ++e) seen[e] = !MASKED || blk + 8 * cq + e <= last;   // what a row does not see may hold anything
            auto weights = [&](auto above) {                       // P and P s of the scores above the reference
                float top = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float a = above(e);
                    p[e] = __builtin_amdgcn_exp2f(seen[e] ? a : -INFINITY);
                    pv[e] = p[e] * (seen[e] ? vs[e] : 0.f);
                    top = fmaxf(top, pv[e]);
                }
                if (tiny)
#pragma unroll
                    for (int e = 0; e < 8; ++e) top = fmaxf(top, p[e] * 0x1p-60f);
                return top;
            };
            const float top =
                weights([&](int e) { return __builtin_fmaf(ks[e], st[mt][e >> 2][e & 3], __builtin_fmaf(kz[e], qsum[mt], -ref[mt])); });
            // (infinite references, of infinite scores, stay)
            if (__builtin_amdgcn_ballot_w64(top > limit && ref[mt] < INFINITY)) {
                if (apart) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) st[mt][e >> 2][e & 3] = st[mt][e >> 2][e & 3] * 16777216.f * s_back[w][mt][lr];
                }
                // Here a score is rounded before the reference leaves it.  Past 2^20 units in the last place are no small
                // part of P's range, so with a bound of that size every tile of the wave comes this way from then on
                float sc[8], bm = KV4_REF0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float v = vs[e];
                    asm volatile("" : "+v"(v));                    // keeps the logarithms on this path
                    sc[e] = __builtin_fmaf(ks[e], st[mt][e >> 2][e & 3], kz[e] * qsum[mt]);
                    if (seen[e]) bm = fmaxf(bm, sc[e] + fmaxf(__builtin_amdgcn_logf(v), -60.f));
                }
                bm = across_rows(bm, [](float a, float b) { return fmaxf(a, b); });
                if (__builtin_amdgcn_ballot_w64(fabsf(bm) > 0x1p20f && bm > KV4_REF0)) limit = -1.f;
                const float to = bm > ref[mt] + 15.f ? bm - 7.f : ref[mt];
                const float corr = to == ref[mt] ? 1.f : __builtin_amdgcn_exp2f(ref[mt] - to);
                ref[mt] = to;
                lsum[mt] *= corr;
                zsum[mt] *= corr;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    oc[mt][i] *= corr;
#pragma unroll
                    for (int nb = 0; nb < NBD; ++nb) o[mt][nb][i] *= corr;
                }
                weights([&](int e) { return sc[e] - ref[mt]; });
                if (limit < 0.f) {                                 // what the reference's own rounding leaves above
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        p[e] = pv[e] > 32768.f ? 32768.f * __builtin_amdgcn_rcpf(vs[e]) : p[e];
                        pv[e] = fminf(pv[e], 32768.f);
                    }
                }
            }
            float2v pr[4];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                lsum[mt] += p[e];
                zsum[mt] = __builtin_fmaf(p[e], seen[e] ? vz[e] : 0.f, zsum[mt]);
                pr[e >> 1][e & 1] = pv[e];
            }
            u32x4 pk;
#pragma unroll
            for (int e = 0; e < 4; ++e) pk[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pr[e], half2v));
            pf[mt] = __builtin_bit_cast(half8, pk);
        }
#pragma unroll
        for (int e = 0; e < NBD; e += 4) *(u32x4*)(vc + e) = *(const u32x4*)(t + 16 * D + 256 * e + 16 * lane);
        __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int nb = 0; nb < NBD; ++nb) {
            const half8 vt = codes(vc[nb]);
#pragma unroll
            for (int mt = 0; mt < MQ; ++mt) o[mt][nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vt, pf[mt], o[mt][nb], 0, 0, 0);
        }
        const half8 mid = codes(0x88888888u);
#pragma unroll
        for (int mt = 0; mt < MQ; ++mt) oc[mt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(mid, pf[mt], oc[mt], 0, 0, 0);
    };
    // a tile waits for its own pieces; once it is used, its place is filled with the tile RING further
    auto tile = [&](int i, auto masked, bool use) {
        if (nt - 1 - i >= AHEAD - 1) wait_tiles<PIECES * (AHEAD - 1)>();
        else wait_tiles<0>();
        if constexpr (ROWS) {
            lds_barrier();                                         // everyone's pieces are in, and the last tile is done with
            if (i + AHEAD < nt) issue(i + AHEAD, (i + AHEAD) % RING);
        }
        if (use && there >> (i & 31) & 1) block(wq0 + STEP * place(i), slots_at + i % RING * SLOT, masked);   // else no page: nothing to see
        if constexpr (!ROWS) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // read before the place is filled again
            if (i + AHEAD < nt) issue(i + AHEAD, i % RING);
        }
    };
    // the tiles that every row sees as a whole, then the others
    int i = 0;
    for (; i < whole; ++i) tile(i, std::false_type(), true);
    for (; i < nt; ++i) tile(i, std::true_type(), i < own);

#pragma unroll
    for (int mt = 0; mt < MQ; ++mt) {
        lsum[mt] += __shfl_xor(lsum[mt], 16, WAVE);
        lsum[mt] += __shfl_xor(lsum[mt], 32, WAVE);
        zsum[mt] += __shfl_xor(zsum[mt], 16, WAVE);
        zsum[mt] += __shfl_xor(zsum[mt], 32, WAVE);
    }
    // four of row lr's sums, the dims NBD (4 cq + i) + nb + 0..3
    auto sums = [&](int mt, int i, int nb) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(o[mt][nb + e][i] - oc[mt][i], 16777216.f, zsum[mt]);
        return make_float4(v[0], v[1], v[2], v[3]);
    };
    // dims d.. of a row of the slice: to the partial results, or the output itself
    auto put = [&](int qrow, int d, float top, float l, float4 x) {
        if (qrow >= QR) return;
        if (it.nch > 1) {
            float* pp = part + part_at(item, n_kv, kvh, G * r.n, qrow, D);
            if (d == 0) *(float2*)pp = make_float2(top, l);
            *(float4*)(pp + 4 + d) = x;
            return;
        }
        const int i = qrow / G, h = qrow - i * G;
        kv4_store4(out, out_t, (size_t)(row0 + i) * out_ld + (size_t)(kvh * G + h) * D + d,
                   l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(x.x / l, x.y / l, x.z / l, x.w / l));
    };
    if constexpr (ROWS) {
#pragma unroll
        for (int mt = 0; mt < MQ; ++mt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int nb = 0; nb < NBD; nb += 4)
                    put(qbase + 16 * mt + lr, NBD * (4 * cq + i) + nb, ref[mt], lsum[mt], sums(mt, i, nb));
        return;
    }
    // merge the four waves, 16 query rows at a time
    float (*s_o)[16 * LDO] = (float (*)[16 * LDO])s_buf;
#pragma unroll
    for (int mt = 0; mt < MQ; ++mt) {
        __syncthreads();
        if (cq == 0) { s_ml[w][0][lr] = ref[mt]; s_ml[w][1][lr] = lsum[mt]; }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int nb = 0; nb < NBD; nb += 4) *(float4*)(&s_o[w][lr * LDO + NBD * (4 * cq + i) + nb]) = sums(mt, i, nb);
        __syncthreads();
        for (int idx = threadIdx.x; idx < 16 * D / 4; idx += 256) {
            const int qr = idx / (D / 4), d = 4 * (idx - qr * (D / 4));
            float mm = s_ml[0][0][qr];
#pragma unroll
            for (int ww = 1; ww < 4; ++ww) mm = fmaxf(mm, s_ml[ww][0][qr]);
            float ls = 0.f;
            float4 os = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int ww = 0; ww < 4; ++ww) {
                const float mw = s_ml[ww][0][qr], f = mw == mm ? 1.f : __builtin_amdgcn_exp2f(mw - mm);
                const float4 x = *(const float4*)(&s_o[ww][qr * LDO + d]);
                ls += s_ml[ww][1][qr] * f;
                os = make_float4(os.x + x.x * f, os.y + x.y * f, os.z + x.z * f, os.w + x.w * f);
            }
            put(qbase + 16 * mt + qr, d, mm, ls, os);
        }
    }
}

// The items of a sequence merged: a work-group takes one row and head, D/4 lanes an
// item, so 1024/D items at a time; its partial sums are added in a fixed order.
// One round trip to memory is all it takes up to 8 * 1024/D items (one sequence's
// 64 items 4.6 us, by one thread a dim 21), most of it the launch.
template <int D>
__global__ void __launch_bounds__(256) k_kv4_combine(rows_t r, att_plan plan, int n_q, int n_kv, const float* part,
                                                     void* out, int out_t, long long out_ld)
{
    constexpr int D4 = D / 4, NG = 256 / D4, CB = 8;              // lanes an item, items at a time, loads in flight
    __shared__ float2 s_ml[NG];
    __shared__ float4 s_o[NG][D4];
    const int idx = blockIdx.x / n_q, hq = blockIdx.x - idx * n_q, b = idx / r.n, i = idx - b * r.n;
    const int nlive = r.lim ? min(r.lim[b], r.n) : r.n;
    if (i >= nlive) return;
    const size_t row = r.row0 ? r.row0[b] + i : idx;
    const int2 sq = plan.seq[b];
    const int nch = sq.y;
    if (nch <= 1) return;                                         // the attention wrote the output
    const int G = n_q / n_kv, QR = G * r.n, kvh = hq / G, d4 = threadIdx.x % D4, gp = threadIdx.x / D4;
    const float* pp = part + part_at(sq.x, n_kv, kvh, QR, i * G + hq - kvh * G, D);
    const size_t st = (size_t)n_kv * QR * (D + 4);                // to the next item
    float mm = KV4_REF0, ls = 0.f;
    float4 os = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float m, float l, float4 x) {
        const float f = m == mm ? 1.f : __builtin_amdgcn_exp2f(m - mm);
        ls += l * f;
        os = make_float4(os.x + x.x * f, os.y + x.y * f, os.z + x.z * f, os.w + x.w * f);
    };
    auto raise_to = [&](float m) {
        const float f = mm == m ? 1.f : __builtin_amdgcn_exp2f(mm - m);
        ls *= f;
        os = make_float4(os.x * f, os.y * f, os.z * f, os.w * f);
        mm = m;
    };
    for (int c0 = gp; c0 < nch; c0 += CB * NG) {
        float2 ml[CB];
        float4 x[CB];
#pragma unroll
        for (int u = 0; u < CB; ++u) {
            const float* pc = pp + min(c0 + u * NG, nch - 1) * st;
            ml[u] = *(const float2*)pc;
            x[u] = *(const float4*)(pc + 4 + 4 * d4);
        }
        float bm = mm;
#pragma unroll
        for (int u = 0; u < CB; ++u) bm = fmaxf(bm, ml[u].x);
        raise_to(bm);
#pragma unroll
        for (int u = 0; u < CB; ++u)
            if (c0 + u * NG < nch) add(ml[u].x, ml[u].y, x[u]);
    }
    if (d4 == 0) s_ml[gp] = make_float2(mm, ls);
    s_o[gp][d4] = os;
    __syncthreads();
    if (gp) return;
    float bm = mm;
#pragma unroll
    for (int u = 1; u < NG; ++u) bm = fmaxf(bm, s_ml[u].x);
    raise_to(bm);
#pragma unroll
    for (int u = 1; u < NG; ++u) add(s_ml[u].x, s_ml[u].y, s_o[u][d4]);
    const float4 v = ls == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(os.x / ls, os.y / ls, os.z / ls, os.w / ls);
    kv4_store4(out, out_t, row * out_ld + (size_t)hq * D + 4 * d4, v);
}

// NaN groups in the positions [kv_len, kv_len + span) of every layer and KV head
__global__ void __launch_bounds__(256) k_kv4_poison(const int32_t* slots, const int32_t* kv_len, int span, kv4_geom g,
                                                    int n_layers, int n_kv, int D, int max_slots, int max_ctx)
{
    const int s = slots[blockIdx.x];
    if (s < 0 || s >= max_slots) return;
    const int lo = max(kv_len[s], 0), per = max((int)min((long long)lo + span, (long long)max_ctx) - lo, 0);
    const long long total = (long long)n_layers * n_kv * per;
    for (long long t = threadIdx.x; t < total; t += 256) {
        const int lh = (int)(t / per), l = lh / n_kv, h = lh - l * n_kv, p = lo + (int)(t - (long long)lh * per);
        const int pg = kv4_page(g, s, p / g.P);
        if (pg < 0) continue;
        uint8_t* tile = g.pages + pg * g.PS + l * g.LS + h * g.HS + (size_t)((p % g.P) >> 5) * tile_bytes(D);
        ((uint32_t*)(tile + 32 * D))[p & 31] = 0x7fc07fc0u;
        ((uint32_t*)(tile + 32 * D + 128))[p & 31] = 0x7fc07fc0u;
    }
}

}  // namespace

// ======================================================================= launchers
void launch_rope_table(const sd_rope_cfg& c, int n_pos, float* table, hipStream_t s)
{
    double lo = 0, hi = 0, mul = 1;
    if (c.scaling == SD_ROPE_YARN) {
        auto at = [&](double turns) { return c.rot_dim * log(c.orig_ctx / (6.283185307179586 * turns)) / (2 * log(c.theta)); };
        lo = fmax(floor(at(c.high)), 0.0);
        hi = fmin(ceil(at(c.low)), c.rot_dim - 1.0);
        mul = c.attn_factor > 0 ? c.attn_factor : 0.1 * log(c.factor) + 1.0;
    }
    auto blocks = [&](int fine) { return (n_pos + fine * fine - 1) / (fine * fine); };
    // from 256 groups of the larger kind on, one a CU
    if (blocks(16) >= 256) k_rope_table<16><<<blocks(16), 512, 0, s>>>(c, lo, hi, mul, n_pos, (float2*)table);
    else k_rope_table<8><<<blocks(8), 512, 0, s>>>(c, lo, hi, mul, n_pos, (float2*)table);
}

template <typename T>
void launch_kv4_append(const rows_t& r, const kv4_geom& g, int n_q, int n_kv, int D, kv4_src<T> k, kv4_src<T> v, kv4_src<T> q,
                       uint16_t* q_out, const kv4_rope& ro, hipStream_t s)
{
    const int ngr = (r.n + 14) / 8;                               // groups of 8 that n rows can touch
    // KV heads a wave: one, or as many as leave KV4_APPEND_WAVES waves
    const long long one = (long long)r.B * ngr * 2 * n_kv;
    int hpw = one > KV4_APPEND_WAVES ? (int)min((long long)n_kv, one / KV4_APPEND_WAVES) : 1;
    const int hw = (n_kv + hpw - 1) / hpw;
    hpw = (n_kv + hw - 1) / hw;                                   // evenly
    const long long kvw = (long long)r.B * ngr * 2 * ((n_kv + hpw - 1) / hpw), qh = q_passes<T>() * 512 / D;
    const long long qw = q_out ? (long long)r.B * r.n * ((n_q + qh - 1) / qh) : 0;
    const unsigned blocks = (unsigned)((kvw + qw + 3) / 4);
    if (D == 128) k_kv4_append<T, 128><<<blocks, 256, 0, s>>>(r, g, n_q, n_kv, k, v, q, q_out, ro, ngr, hpw, (int)kvw);
    else k_kv4_append<T, 64><<<blocks, 256, 0, s>>>(r, g, n_q, n_kv, k, v, q, q_out, ro, ngr, hpw, (int)kvw);
}
template void launch_kv4_append<float>(const rows_t&, const kv4_geom&, int, int, int, kv4_src<float>, kv4_src<float>,
                                       kv4_src<float>, uint16_t*, const kv4_rope&, hipStream_t);
template void launch_kv4_append<f32_parts>(const rows_t&, const kv4_geom&, int, int, int, kv4_src<f32_parts>, kv4_src<f32_parts>,
                                           kv4_src<f32_parts>, uint16_t*, const kv4_rope&, hipStream_t);
template void launch_kv4_append<uint16_t>(const rows_t&, const kv4_geom&, int, int, int, kv4_src<uint16_t>, kv4_src<uint16_t>,
                                          kv4_src<uint16_t>, uint16_t*, const kv4_rope&, hipStream_t);

void launch_kv4_read(const rows_t& r, const kv4_geom& g, int n_kv, int D, const int32_t* start, uint16_t* k_out,
                     uint16_t* v_out, hipStream_t s)
{
    const int ngr = (r.n + 14) / 8;
    const long long total = (long long)r.B * ngr * 2 * n_kv * (D / 8);
    const unsigned blocks = (unsigned)((total + 255) / 256);
    if (D == 128) k_kv4_read<128><<<blocks, 256, 0, s>>>(r, g, n_kv, k_out, v_out, start, ngr, total);
    else k_kv4_read<64><<<blocks, 256, 0, s>>>(r, g, n_kv, k_out, v_out, start, ngr, total);
}

template <int D>
static void kv4_attn_d(const rows_t& r, const att_plan& pl, const kv4_geom& g, int n_q, int n_kv, const uint16_t* q,
                       long long q_ld, float cs, float* part, void* out, act_t out_t, long long out_ld, hipStream_t s,
                       hipEvent_t ev0, hipEvent_t ev1)
{
    auto go = [&](auto kern) {
        const dim3 grid(n_kv, pl.max_items, pl.zs), block(256);
        if (ev0) hipExtLaunchKernelGGL(kern, grid, block, 0, s, ev0, ev1, 0, r, g, n_q, n_kv, q, q_ld, cs, part, pl, out, (int)out_t, out_ld);
        else kern<<<grid, block, 0, s>>>(r, g, n_q, n_kv, q, q_ld, cs, part, pl, out, (int)out_t, out_ld);
    };
    if (pl.mq == 1) go(pl.by_rows ? k_kv4_attn<D, 1, true> : k_kv4_attn<D, 1, false>);
    else go(pl.by_rows ? k_kv4_attn<D, 2, true> : k_kv4_attn<D, 2, false>);
}

void launch_kv4_attention(const rows_t& r, const att_plan& pl, const kv4_geom& g, int n_q, int n_kv, int D, const uint16_t* q,
                          long long q_ld, float scale, float* part, void* out, act_t out_t, long long out_ld, hipStream_t s,
                          hipEvent_t ev0, hipEvent_t ev1)
{
    const float cs = (float)(scale * 1.4426950408889634);
    if (D == 128) kv4_attn_d<128>(r, pl, g, n_q, n_kv, q, q_ld, cs, part, out, out_t, out_ld, s, ev0, ev1);
    else kv4_attn_d<64>(r, pl, g, n_q, n_kv, q, q_ld, cs, part, out, out_t, out_ld, s, ev0, ev1);
}

void launch_kv4_combine(const rows_t& r, const att_plan& pl, int n_q, int n_kv, int D, const float* part, void* out,
                        act_t out_t, long long out_ld, hipStream_t s)
{
    if (D == 128) k_kv4_combine<128><<<r.B * r.n * n_q, 256, 0, s>>>(r, pl, n_q, n_kv, part, out, (int)out_t, out_ld);
    else k_kv4_combine<64><<<r.B * r.n * n_q, 256, 0, s>>>(r, pl, n_q, n_kv, part, out, (int)out_t, out_ld);
}

void launch_kv4_poison(int B, const int32_t* slots, const int32_t* kv_len, int span, const kv4_geom& g, int n_layers, int n_kv,
                       int D, int max_slots, int max_ctx, hipStream_t s)
{
    k_kv4_poison<<<B, 256, 0, s>>>(slots, kv_len, span, g, n_layers, n_kv, D, max_slots, max_ctx);
}
