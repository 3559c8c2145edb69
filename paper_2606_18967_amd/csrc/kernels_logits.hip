// kernels_logits.hip -- what a learner needs of logits rows: the tokens'
// log-probabilities, the rows' entropies, their gradients, and the clipped
// policy loss with its gradient.
//
// With x a row of V logits, m its largest and c = log2(e)/T, everything follows
// from sums over e_j = 2^(y_j), y_j = c (x_j - m) <= 0:
//   s = sum e_j,  t = sum e_j y_j:
//   ln p_j = ln2 (y_j - log2 s),   H = ln2 (log2 s - t/s),
// and the gradient of g ln p_tok + h H with respect to x_j is
//   (g [j = tok] - e_j (a + b y_j))/T,  a = (g + h (H - ln s))/s,  b = h ln2/s.
// The difference is taken before the product: it is exact or off by 2^-24 of itself,
// whatever the logits' common offset (c x - c m in one fused operation is off by
// 2^-24 of c m, and far out of range for equal logits of 1e30).  All sums
// are fp32 in a fixed order (the loss's sums over the rows fp64); a bf16
// gradient is rounded once.  A logit of -inf has p = 0 and no gradient; where y
// is a factor it is held above Y_MIN, so that 0 y is 0.
//
// What bounds them: the bytes of the logits.  A gradient needs its row's sums first;
// where one kernel makes both, the second reading is left to the caches, and all
// others go past them: the loss of 8192 x 128256 bf16 rows (a fifth of them padding,
// 3.8 GB of logits and gradients) takes 735 us, which is the rate of a large copy,
// with both readings past the caches 958, with neither 746, with work-groups of 512
// threads instead of 1024 767.  The log-probabilities of 2048 x 152064 and their
// gradient, two readings and a writing, take 322 us (5.8 TB/s; 340 where the gradient
// is stored through the caches, which the next kernel has to wait for).
#include "common.h"
#include "kernels.h"

namespace {

constexpr float LN2 = 0.6931471805599453f;
constexpr float Y_MIN = -1e4f;              // 2^Y_MIN = 0

// eight or four logits as they lie in memory, at any element's alignment
template <typename T> struct pack_t;
template <> struct pack_t<uint16_t> {
    static constexpr int N = 8;
    typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(2)));
    static __device__ __forceinline__ void get(u32x4 w, float (&x)[N])
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[2 * e] = __uint_as_float(w[e] << 16);
            x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ u32x4 put(const float (&x)[N])
    {
        return (u32x4){pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
    }
};
template <> struct pack_t<float> {
    static constexpr int N = 4;
    typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(4)));
    static __device__ __forceinline__ void get(u32x4 w, float (&x)[N])
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(w[e]);
    }
    static __device__ __forceinline__ u32x4 put(const float (&x)[N])
    {
        return (u32x4){__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    }
};

// KEEP: the logits are read again, and are to stay in the caches until then
template <bool KEEP, typename T>
__device__ __forceinline__ u32x4 load_vec(const T* p)
{
    const auto v = (const typename pack_t<T>::vec*)p;
    return KEEP ? (u32x4)*v : (u32x4)__builtin_nontemporal_load(v);
}
template <typename T>
__device__ __forceinline__ void store_vec(T* p, u32x4 v)
{
    __builtin_nontemporal_store((typename pack_t<T>::vec)v, (typename pack_t<T>::vec*)p);
}

// running sums of a part of a row: m the largest logit, s and t as above
struct part_t { float m, s, t; };

// what to subtract where nothing but -inf was met
__device__ __forceinline__ float origin(float m) { return m == -INFINITY ? 0.f : m; }

template <int N>
__device__ __forceinline__ void take(part_t& a, const float (&x)[N], float m, float c)
{
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float y = (x[e] - m) * c, p = __builtin_amdgcn_exp2f(y);
        a.s += p;
        a.t = __builtin_fmaf(p, fmaxf(y, Y_MIN), a.t);
    }
}
// the sums moved to the largest logit m, which is not below their own (so d <= 0, -inf among it; where they met nothing but
// -inf they are 0, or NaN and stay so)
__device__ __forceinline__ void move_to(part_t& a, float m, float c)
{
    const float d = a.m == -INFINITY ? 0.f : (a.m - m) * c, f = __builtin_amdgcn_exp2f(d);
    a.t = (a.t + fmaxf(d, Y_MIN) * a.s) * f;
    a.s *= f;
    a.m = m;
}

// the parts of a work-group's threads joined, in every thread; sh: 3 * 16 floats
__device__ __forceinline__ part_t join(part_t a, float c, float* sh)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
    float m = wave_max(a.m);
    if (nw > 1) {
        if (lane == 0) sh[w] = m;
        __syncthreads();
        for (int i = 0; i < nw; ++i) m = fmaxf(m, sh[i]);
    }
    // a part without a finite logit has s = t = 0 or, from a NaN or +inf, NaN
    if (a.m > -INFINITY) move_to(a, m, c);
    a.m = m;
    a.s = wave_sum(a.s);
    a.t = wave_sum(a.t);
    if (nw > 1) {
        if (lane == 0) { sh[16 + w] = a.s; sh[32 + w] = a.t; }
        __syncthreads();
        a.s = a.t = 0.f;
        for (int i = 0; i < nw; ++i) { a.s += sh[16 + i]; a.t += sh[32 + i]; }
    }
    return a;
}

// A thread's pass over the logits [from, n) of a row part, vector by vector of the
// work-group, U of them under way at once.
template <typename T, int U, bool KEEP>
__device__ __forceinline__ void sum_part(part_t& a, const T* x, int first, int n, float c)
{
    constexpr int N = pack_t<T>::N;
    const int step = blockDim.x * N;
    for (int i0 = first + threadIdx.x * N; i0 + N <= n; i0 += U * step) {
        u32x4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = load_vec<KEEP>(x + min(i0 + u * step, n - N));
        float m = a.m, y[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            pack_t<T>::get(v[u], y[u]);
            if (i0 + u * step + N > n) continue;
#pragma unroll
            for (int e = 0; e < N; ++e) m = fmaxf(m, y[u][e]);
        }
        if (m > a.m) move_to(a, m, c);
        const float o = origin(m);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i0 + u * step + N <= n) take<N>(a, y[u], o, c);
    }
}
// the last n % N logits of a row part that starts at a whole vector: one of the first threads each
template <typename T>
__device__ __forceinline__ void sum_tail(part_t& a, const T* x, int n, float c)
{
    constexpr int N = pack_t<T>::N;
    const int i = n / N * N + threadIdx.x;
    if (i >= n) return;
    const float v[1] = {elem<T>::load(x, i)};
    if (v[0] > a.m) move_to(a, v[0], c);
    take<1>(a, v, origin(a.m), c);
}

// what a row's sums give its token
struct row_stat { float logp, entropy, ln_s; };
__device__ __forceinline__ row_stat row_of(const part_t& a, float xt, float T)
{
    row_stat r;
    r.ln_s = log2f(a.s) * LN2;
    r.logp = (xt - a.m) / T - r.ln_s;
    r.entropy = r.ln_s - a.t / a.s * LN2;
    return r;
}

// the gradient's factors: d_j = e_j (A + B y_j), and D added at the token
struct grad_t { float m, A, B, D; };
// q = 1/(s T)
__device__ __forceinline__ grad_t grad_of(float m, float ln_s, float q, float entropy, float g, float h, float T)
{
    return grad_t{origin(m), -(g + (h != 0.f ? h * (entropy - ln_s) : 0.f)) * q, -h * LN2 * q, g / T};
}
template <bool ENT>
__device__ __forceinline__ float grad_at(float x, const grad_t& d, float c)
{
    const float y = (x - d.m) * c, e = __builtin_amdgcn_exp2f(y);
    return e * (ENT ? __builtin_fmaf(d.B, fmaxf(y, Y_MIN), d.A) : d.A);
}

template <bool ENT, int N>
__device__ __forceinline__ void grad_vec(float (&x)[N], const grad_t& d, float c)
{
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = grad_at<ENT>(x[e], d, c);
}

// A thread's pass that writes the gradient of the logits [first, n), and of the last
// n % N where tail is set.  out may be x: a thread reads what it writes first.
template <typename T, bool ENT, int U>
__device__ __forceinline__ void grad_part(const T* x, T* out, int first, int n, const grad_t& d, float c)
{
    constexpr int N = pack_t<T>::N;
    const int step = blockDim.x * N;
    for (int i0 = first + threadIdx.x * N; i0 + N <= n; i0 += U * step) {
        u32x4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i0 + u * step + N <= n) v[u] = load_vec<false>(x + i0 + u * step);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u * step + N > n) break;
            float y[N];
            pack_t<T>::get(v[u], y);
            grad_vec<ENT>(y, d, c);
            store_vec(out + i0 + u * step, pack_t<T>::put(y));
        }
    }
}
template <typename T, bool ENT>
__device__ __forceinline__ void grad_tail(const T* x, T* out, int n, const grad_t& d, float c)
{
    const int i = n / pack_t<T>::N * pack_t<T>::N + threadIdx.x;
    if (i < n) elem<T>::store(out, i, grad_at<ENT>(elem<T>::load(x, i), d, c));
}
template <typename T>
__device__ __forceinline__ void zero_part(T* out, int n)
{
    constexpr int N = pack_t<T>::N;
    for (int i = threadIdx.x * N; i + N <= n; i += blockDim.x * N) store_vec(out + i, (u32x4){0, 0, 0, 0});
    const int i = n / N * N + threadIdx.x;
    if (i < n) elem<T>::store(out, i, 0.f);
}

// ------------------------------------------------------------------ rows of the policy loss
// A row that counts: weight, a token of the vocabulary, an importance ratio inside
// the filter.  drop: it has a weight but is filtered.
struct live_t { bool live, drop; };
__device__ __forceinline__ live_t policy_live(const policy_args& p, int row, int V)
{
    const float w = p.weight[row];
    const int tok = p.tok[row];
    if (!(w != 0.f) || tok < 0 || tok >= V) return {false, false};
    if (!p.behavior) return {true, false};
    const float far = p.old_logp[row] - p.behavior[row];
    const bool in = far >= p.log_is_low && far <= p.log_is_high;
    return {in, !in};
}

// The row's terms of the loss, and the gradients of the loss by its ln p and H
struct policy_row { float term[POLICY_TERMS], g, h; };
__device__ __forceinline__ policy_row policy_of(const policy_args& p, int row, const row_stat& st)
{
    const float w = p.weight[row], A = p.adv[row], far = st.logp - p.old_logp[row], r = expf(far);
    // (r may be past fp32's range, and 0 times it is 0 all the same)
    const float free = A == 0.f && fabsf(far) < INFINITY ? 0.f : r * A;
    const float cut = fminf(fmaxf(r, 1.f - p.clip_low), 1.f + p.clip_high) * A;
    const bool clipped = cut < free;
    const float pg = -(clipped ? cut : free);                   // a NaN ratio or advantage stays one
    float kl = 0.f, dkl = 0.f;
    if (p.ref_logp) {                                           // e^x - x - 1 and -(e^x - 1), x = ref - logp
        const float x = p.ref_logp[row] - st.logp, em = expm1f(x);
        kl = em - x;
        dkl = -em;
    }
    policy_row o;
    // (a term that the loss does not have may be infinite or NaN)
    const float klw = p.kl_coef != 0.f ? p.kl_coef * kl : 0.f, dklw = p.kl_coef != 0.f ? p.kl_coef * dkl : 0.f;
    const float entw = p.entropy_coef != 0.f ? p.entropy_coef * st.entropy : 0.f;
    o.term[0] = w * (pg + klw - entw);
    o.term[1] = w * pg;
    o.term[2] = w * kl;
    o.term[3] = w * st.entropy;
    o.term[4] = clipped ? w : 0.f;
    o.term[5] = 0.f;
    o.g = w * ((clipped ? 0.f : -free) + dklw);
    o.h = -p.entropy_coef * w;
    return o;
}

__device__ __forceinline__ void dead_row(const policy_args& p, int row, bool drop)
{
    p.logp[row] = 0.f;
    if (p.entropy) p.entropy[row] = 0.f;
    for (int k = 0; k < POLICY_TERMS; ++k) p.terms[(size_t)row * POLICY_TERMS + k] = 0.f;
    if (drop) p.terms[(size_t)row * POLICY_TERMS + 5] = p.weight[row];
}
__device__ __forceinline__ void put_row(const policy_args& p, int row, const row_stat& st, const policy_row& o)
{
    p.logp[row] = st.logp;
    if (p.entropy) p.entropy[row] = st.entropy;
    for (int k = 0; k < POLICY_TERMS; ++k) p.terms[(size_t)row * POLICY_TERMS + k] = o.term[k];
}

// A work-group a row: its sums, the token's terms, and the gradient.
template <typename T, bool ENT, bool GRAD>
__global__ void __launch_bounds__(1024) k_policy_rows(logits_args a, policy_args p)
{
    __shared__ float sh[48];
    const int row = blockIdx.x, V = a.V;
    const T* x = (const T*)a.x + (long long)row * a.ld;
    T* out = GRAD ? (T*)a.out + (long long)row * a.out_ld : nullptr;
    const live_t lv = policy_live(p, row, V);
    if (!lv.live) {
        if (threadIdx.x == 0) dead_row(p, row, lv.drop);
        if (GRAD) zero_part(out, V);
        return;
    }
    const int tok = p.tok[row];
    const float xt = elem<T>::load(x, tok);
    part_t s = {-INFINITY, 0.f, 0.f};
    sum_part<T, 4, GRAD>(s, x, 0, V, a.c);
    sum_tail(s, x, V, a.c);
    s = join(s, a.c, sh);
    const row_stat st = row_of(s, xt, a.T);
    const policy_row o = policy_of(p, row, st);
    if (threadIdx.x == 0) put_row(p, row, st, o);
    if (GRAD) {
        const grad_t d = grad_of(s.m, st.ln_s, 1.f / (s.s * a.T), st.entropy, o.g, o.h, a.T);
        grad_part<T, ENT, 4>(x, out, 0, V, d, a.c);
        grad_tail<T, ENT>(x, out, V, d, a.c);
        // the token's own, by the thread that wrote its place before
        constexpr int N = pack_t<T>::N;
        const int body = V / N * N;
        if (threadIdx.x == (tok < body ? tok / N % blockDim.x : tok - body))
            elem<T>::store(out, tok, grad_at<ENT>(xt, d, a.c) + d.D);
    }
}

// A row in several work-groups, where there are few rows: the sums of a part each, and the token's logit, over which a
// gradient may be written before the last part has read it.
template <typename T, bool KEEP>
__global__ void __launch_bounds__(256) k_row_parts(logits_args a, const int32_t* tok, part_t* parts, float* at_tok)
{
    __shared__ float sh[48];
    const int row = blockIdx.y, k = blockIdx.x, c0 = k * a.chunk, n = min(a.chunk, a.V - c0);
    if (tok[row] < 0 || tok[row] >= a.V) return;
    const T* x = (const T*)a.x + (long long)row * a.ld + c0;
    part_t s = {-INFINITY, 0.f, 0.f};
    sum_part<T, 4, KEEP>(s, x, 0, n, a.c);
    sum_tail(s, x, n, a.c);
    s = join(s, a.c, sh);
    if (threadIdx.x == 0) {
        parts[(size_t)row * gridDim.x + k] = s;
        const int at = tok[row] - c0;
        if (at >= 0 && at < n) at_tok[row] = elem<T>::load(x, at);
    }
}
// the parts of a row joined by one wave, in every lane
__device__ __forceinline__ part_t join_parts(const part_t* parts, int row, int S, float c)
{
    const int lane = threadIdx.x & 63;
    part_t a = {-INFINITY, 0.f, 0.f};
    for (int k = lane; k < S; k += WAVE) {
        part_t b = parts[(size_t)row * S + k];
        if (b.m > a.m) move_to(a, b.m, c);
        else if (b.m > -INFINITY) move_to(b, a.m, c);
        a.s += b.s;
        a.t += b.t;
    }
    const float m = wave_max(a.m);
    if (a.m > -INFINITY) move_to(a, m, c);
    a.m = m;
    a.s = wave_sum(a.s);
    a.t = wave_sum(a.t);
    return a;
}

// ------------------------------------------------------------------ log-probabilities
__device__ __forceinline__ void put_logp(const logp_args& p, int row, const part_t& s, const row_stat& st, bool live)
{
    p.logp[row] = live ? st.logp : 0.f;
    if (p.entropy) p.entropy[row] = live ? st.entropy : 0.f;
    if (p.norm) {
        p.norm[2 * (size_t)row] = live ? s.m : 0.f;
        p.norm[2 * (size_t)row + 1] = live ? st.ln_s : 0.f;
    }
}
template <typename T>
__global__ void __launch_bounds__(1024) k_logp_rows(logits_args a, logp_args p)
{
    __shared__ float sh[48];
    const int row = blockIdx.x, V = a.V, tok = p.tok[row];
    const T* x = (const T*)a.x + (long long)row * a.ld;
    part_t s = {-INFINITY, 0.f, 0.f};
    const bool live = tok >= 0 && tok < V;
    float xt = 0.f;
    if (live) {
        xt = elem<T>::load(x, tok);
        sum_part<T, 4, false>(s, x, 0, V, a.c);
        sum_tail(s, x, V, a.c);
        s = join(s, a.c, sh);
    }
    if (threadIdx.x == 0) put_logp(p, row, s, row_of(s, xt, a.T), live);
}
__global__ void __launch_bounds__(64) k_logp_finish(logits_args a, logp_args p, const part_t* parts, int S, const float* at_tok)
{
    const int row = blockIdx.x, tok = p.tok[row];
    const bool live = tok >= 0 && tok < a.V;
    part_t s = {-INFINITY, 0.f, 0.f};
    float xt = 0.f;
    if (live) {
        xt = at_tok[row];
        s = join_parts(parts, row, S, a.c);
    }
    if (threadIdx.x == 0) put_logp(p, row, s, row_of(s, xt, a.T), live);
}

// The gradient of a row part from the row's norm (its largest logit and ln s): one
// pass.
template <typename T, bool ENT>
__global__ void __launch_bounds__(1024) k_logp_grad(logits_args a, logp_grad_args p, int S)
{
    const int row = blockIdx.x / S, k = blockIdx.x - row * S, c0 = k * a.chunk, n = min(a.chunk, a.V - c0), tok = p.tok[row];
    const T* x = (const T*)a.x + (long long)row * a.ld + c0;
    T* out = (T*)a.out + (long long)row * a.out_ld + c0;
    if (tok < 0 || tok >= a.V) {
        zero_part(out, n);
        return;
    }
    const float g = p.dlogp[row], h = ENT ? p.dentropy[row] : 0.f, m = p.norm[2 * (size_t)row], ln_s = p.norm[2 * (size_t)row + 1];
    const grad_t d = grad_of(m, ln_s, expf(-ln_s) / a.T, ENT ? p.entropy[row] : 0.f, g, h, a.T);
    float xt = 0.f;
    const int at = tok - c0;
    if (at >= 0 && at < n) xt = elem<T>::load(x, at);
    constexpr int N = pack_t<T>::N;
    grad_part<T, ENT, 4>(x, out, 0, n, d, a.c);
    grad_tail<T, ENT>(x, out, n, d, a.c);
    const int body = n / N * N;
    if (at >= 0 && at < n && threadIdx.x == (at < body ? at / N % blockDim.x : at - body))
        elem<T>::store(out, at, grad_at<ENT>(xt, d, a.c) + d.D);
}

// ------------------------------------------------------------------ the loss of few rows
// The rows' terms from their parts.
__global__ void __launch_bounds__(64) k_policy_finish(logits_args a, policy_args p, const part_t* parts, int S, const float* at_tok)
{
    const int row = blockIdx.x;
    const live_t lv = policy_live(p, row, a.V);
    if (!lv.live) {
        if (threadIdx.x == 0) dead_row(p, row, lv.drop);
        return;
    }
    const part_t s = join_parts(parts, row, S, a.c);
    const row_stat st = row_of(s, at_tok[row], a.T);
    if (threadIdx.x == 0) put_row(p, row, st, policy_of(p, row, st));
}
// The same with the gradient of a part: every wave joins the row's parts for itself, which costs less than a launch for it.
template <typename T, bool ENT>
__global__ void __launch_bounds__(256) k_policy_grad(logits_args a, policy_args p, const part_t* parts, int S, const float* at_tok)
{
    const int row = blockIdx.y, k = blockIdx.x, c0 = k * a.chunk, n = min(a.chunk, a.V - c0);
    const T* x = (const T*)a.x + (long long)row * a.ld + c0;
    T* out = (T*)a.out + (long long)row * a.out_ld + c0;
    const live_t lv = policy_live(p, row, a.V);
    if (!lv.live) {
        if (k == 0 && threadIdx.x == 0) dead_row(p, row, lv.drop);
        zero_part(out, n);
        return;
    }
    const float xt = at_tok[row];
    const part_t s = join_parts(parts, row, S, a.c);
    const row_stat st = row_of(s, xt, a.T);
    const policy_row o = policy_of(p, row, st);
    if (k == 0 && threadIdx.x == 0) put_row(p, row, st, o);
    const grad_t d = grad_of(s.m, st.ln_s, 1.f / (s.s * a.T), st.entropy, o.g, o.h, a.T);
    grad_part<T, ENT, 4>(x, out, 0, n, d, a.c);
    grad_tail<T, ENT>(x, out, n, d, a.c);
    constexpr int N = pack_t<T>::N;
    const int at = p.tok[row] - c0, body = n / N * N;
    if (at >= 0 && at < n && threadIdx.x == (at < body ? at / N % blockDim.x : at - body))
        elem<T>::store(out, at, grad_at<ENT>(xt, d, a.c) + d.D);
}

// stats[k] = sum of the rows' terms k, in fp64 and a fixed order
__global__ void __launch_bounds__(1024) k_policy_sum(const float* terms, int rows, float* stats)
{
    __shared__ double sh[16][POLICY_TERMS];
    double v[POLICY_TERMS] = {};
    for (int r = threadIdx.x; r < rows; r += 1024)
#pragma unroll
        for (int k = 0; k < POLICY_TERMS; ++k) v[k] += terms[(size_t)r * POLICY_TERMS + k];
#pragma unroll
    for (int k = 0; k < POLICY_TERMS; ++k) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) v[k] += __shfl_xor(v[k], o, WAVE);
        if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6][k] = v[k];
    }
    __syncthreads();
    if (threadIdx.x < POLICY_TERMS) {
        double s = 0.0;
        for (int w = 0; w < 16; ++w) s += sh[w][threadIdx.x];
        stats[threadIdx.x] = (float)s;
    }
}

// threads of a work-group that takes a row (part) of n logits
template <typename T>
int row_threads(int n, int most)
{
    const int want = (n / pack_t<T>::N + 63) / 64 * 64;
    return want < 64 ? 64 : want > most ? most : want;
}

template <typename T>
void logp_t(const logits_args& a, const logp_args& p, int rows, int S, float* work, hipStream_t s)
{
    if (S == 1) {
        k_logp_rows<T><<<rows, row_threads<T>(a.V, 1024), 0, s>>>(a, p);
        return;
    }
    float* at_tok = work;
    part_t* parts = (part_t*)(work + rows);
    k_row_parts<T, false><<<dim3(S, rows), row_threads<T>(a.chunk, 256), 0, s>>>(a, p.tok, parts, at_tok);
    k_logp_finish<<<rows, 64, 0, s>>>(a, p, parts, S, at_tok);
}
template <typename T>
void policy_t(const logits_args& a, const policy_args& p, int rows, int S, float* work, float* stats, hipStream_t s)
{
    const bool ent = p.entropy_coef != 0.f;
    if (S == 1) {
        const int nt = row_threads<T>(a.V, 1024);
        if (!a.out) k_policy_rows<T, false, false><<<rows, nt, 0, s>>>(a, p);
        else if (ent) k_policy_rows<T, true, true><<<rows, nt, 0, s>>>(a, p);
        else k_policy_rows<T, false, true><<<rows, nt, 0, s>>>(a, p);
    } else {
        const int nt = row_threads<T>(a.chunk, 256);
        float* at_tok = work;
        part_t* parts = (part_t*)(work + rows);
        const dim3 grid(S, rows);
        if (a.out) k_row_parts<T, true><<<grid, nt, 0, s>>>(a, p.tok, parts, at_tok);
        else k_row_parts<T, false><<<grid, nt, 0, s>>>(a, p.tok, parts, at_tok);
        if (!a.out) k_policy_finish<<<rows, 64, 0, s>>>(a, p, parts, S, at_tok);
        else if (ent) k_policy_grad<T, true><<<grid, nt, 0, s>>>(a, p, parts, S, at_tok);
        else k_policy_grad<T, false><<<grid, nt, 0, s>>>(a, p, parts, S, at_tok);
    }
    k_policy_sum<<<1, 1024, 0, s>>>(p.terms, rows, stats);
}

}  // namespace

// Parts of a row: few long rows take about 1024 work-groups of at least 4096 logits, others one each.  (The loss with its
// gradient, in parts and whole, us a call: 14 x 50257 fp32 20.3 and 17.6, 40 x 100000 bf16 19.5 and 21.3, 14 x 128256
// fp32 19.7 and 25.9, 130 x 128256 bf16 25.4 and 28.8, 200 x 128256 31.4 and 30.8, 416 x 128256 fp32 94.7 and 90.3, 511 x 152064 bf16
// 75 and 68.)
constexpr int PART_ROWS = 160, PART_V = 65536;
static int row_splits(int rows, int V, int* chunk)
{
    *chunk = V;
    if (rows < 1 || rows >= PART_ROWS || V <= PART_V) return 1;
    const int want = (1024 + rows - 1) / rows, most = V / 4096;
    const int S = want < most ? want : most;
    *chunk = ((V + S - 1) / S + 2047) / 2048 * 2048;
    return (V + *chunk - 1) / *chunk;
}

// for up to so many rows: r < PART_ROWS of them have at most 1024 + r - 1 parts, and their tokens' logits
size_t logits_work_floats(int rows, int V)
{
    const size_t split = V <= PART_V ? 0 : rows < PART_ROWS ? rows : PART_ROWS - 1;
    return (size_t)rows * POLICY_TERMS + (split ? 3 * (1024 + split) + split : 0);
}

void launch_token_logprobs(logits_args a, const logp_args& p, int rows, bool f32, float* work, hipStream_t s)
{
    const int S = row_splits(rows, a.V, &a.chunk);
    if (f32) logp_t<float>(a, p, rows, S, work, s);
    else logp_t<uint16_t>(a, p, rows, S, work, s);
}

void launch_token_logprobs_grad(logits_args a, const logp_grad_args& p, int rows, bool f32, hipStream_t s)
{
    const int S = row_splits(rows, a.V, &a.chunk);
    const int grid = S * rows;
    if (f32) {
        const int nt = row_threads<float>(a.chunk, 1024);
        if (p.dentropy) k_logp_grad<float, true><<<grid, nt, 0, s>>>(a, p, S);
        else k_logp_grad<float, false><<<grid, nt, 0, s>>>(a, p, S);
    } else {
        const int nt = row_threads<uint16_t>(a.chunk, 1024);
        if (p.dentropy) k_logp_grad<uint16_t, true><<<grid, nt, 0, s>>>(a, p, S);
        else k_logp_grad<uint16_t, false><<<grid, nt, 0, s>>>(a, p, S);
    }
}

void launch_policy_loss(logits_args a, policy_args p, int rows, bool f32, float* work, float* stats, hipStream_t s)
{
    p.terms = work;
    if (rows == 0) {
        k_policy_sum<<<1, 1024, 0, s>>>(p.terms, 0, stats);
        return;
    }
    const int S = row_splits(rows, a.V, &a.chunk);
    work += (size_t)rows * POLICY_TERMS;
    if (f32) policy_t<float>(a, p, rows, S, work, stats, s);
    else policy_t<uint16_t>(a, p, rows, S, work, stats, s);
}
