// rope_rows.h -- rows of heads as the appends take them: eight dims a lane, from any
// of the sources of kv4_src (kernels.h), rotated by a table.
#pragma once
#include "common.h"
#include "kernels.h"

namespace {

// a first position (kv_len and the like hold anything) kept where sums with row numbers
// stay in 32 bits; past 2^24 either way (the longest cache) no row has a place
__device__ __forceinline__ int kv4_base(long long pos) { return (int)min(max(pos, -(1ll << 25)), 1ll << 25); }

__device__ __forceinline__ void raise(uint32_t* err, int kind)
{
    if (err) flag_error(err, kind);
}

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

}  // namespace
