// What the attention kernels share: head tensors, visible ranges, score functions.
#pragma once

#include "common.cuh"

namespace noble {
namespace attn {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// A tensor of heads (noble_heads), typed.
template <typename T>
struct Heads {
    T *p;
    int64_t row, head;
    __device__ __forceinline__ T *at(int64_t t, int64_t h) const { return p + t * row + h * head; }
};

// Which keys a query sees.  Document, causal, prefix and window masks all leave
// one range [lo, hi) of keys per query, and both ends ascend with the query, so
// the keys of a block of queries are those from its first query's lo to its last
// one's hi, and the queries that see a key are a range too.  Tokens of no document
// get an empty range that keeps the order.
struct Mask {
    const int32_t *doc_start, *prefix;  // prefix NULL: none
    int n_docs, T, window;              // window 0: none
    int causal;
};

struct Range {
    int lo, hi;
};

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }

// Range of query i, 0 <= i < T.  Both ends stay within [0, T].
__device__ __forceinline__ Range visible(const Mask &m, int i)
{
    // the last document that starts at or before i (empty documents share a start)
    int a = -1, b = m.n_docs + 1;
    while (b - a > 1) {
        const int c = (a + b) >> 1;
        if (m.doc_start[c] <= i) a = c;
        else b = c;
    }
    if (a < 0) {
        const int s = clampi(m.doc_start[0], 0, m.T);
        return {s, s};
    }
    const int s = clampi(m.doc_start[a], 0, m.T);
    if (a == m.n_docs) return {s, s};
    const int e = clampi(m.doc_start[a + 1], s, m.T);
    Range r = {s, e};
    if (m.causal) {
        r.hi = i + 1;
        if (m.prefix) r.hi = max(r.hi, s + clampi(m.prefix[a], 0, e - s));
    } else if (m.window) {
        r.hi = min(e, i + m.window);
    }
    if (m.window) r.lo = max(s, i - m.window + 1);
    r.hi = clampi(r.hi, 0, e);
    return r;
}

// One past the last token of a document.
__device__ __forceinline__ int docs_end(const Mask &m) { return clampi(m.doc_start[m.n_docs], 0, m.T); }

// scale q.k -> s (capped, biased), and the derivative of s by its first argument.
struct Score {
    float scale, softcap;  // softcap 0: none
    const float *slope;    // per query head, or NULL
};

// tanh from the exponential: 1 - 2 / (1 + e^2x).  Its error is a rounding of 1, which
// the caller multiplies by the cap, as the rounding of a score near the cap is.
__device__ __forceinline__ float tanh_exp(float x)
{
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x * (2.f * kLog2e)));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return fmaf(-2.f, r, 1.f);
}
__device__ __forceinline__ float exp2_fast(float x)
{
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x));
    return e;
}

__device__ __forceinline__ float load_f(const float *p) { return *p; }
__device__ __forceinline__ float load_f(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_f(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_f(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

// Four consecutive elements (a 16- or 8-byte load or store).
__device__ __forceinline__ float4 load4(const float *p) { return *reinterpret_cast<const float4 *>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16 *p)
{
    const uint2 u = *reinterpret_cast<const uint2 *>(p);
    const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&u.x));
    const float2 b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&u.y));
    return make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ void store4(float *p, float4 v) { *reinterpret_cast<float4 *>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16 *p, float4 v)
{
    __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
    uint2 u;
    u.x = *reinterpret_cast<uint32_t *>(&a);
    u.y = *reinterpret_cast<uint32_t *>(&b);
    *reinterpret_cast<uint2 *>(p) = u;
}

// Eight.
__device__ __forceinline__ void load8(float (&x)[8], const float *p)
{
    const float4 a = load4(p), b = load4(p + 4);
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
__device__ __forceinline__ void load8(float (&x)[8], const __nv_bfloat16 *p)
{
    const uint4 u = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t pack2(float a, float b)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ float sum2(uint64_t v)
{
    float a, b;
    unpack2(v, a, b);
    return a + b;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// 8 elements as they are in memory
template <typename T> struct Raw;
template <> struct Raw<__nv_bfloat16> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const __nv_bfloat16 *p)
    {
        const uint4 u = *reinterpret_cast<const uint4 *>(p);
        w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const { *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]); }
    __device__ __forceinline__ void zero() { w[0] = w[1] = w[2] = w[3] = 0; }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    __device__ __forceinline__ void get(uint64_t (&x)[4]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
    }
    __device__ __forceinline__ Raw from(int lane) const
    {
        Raw r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = __shfl_sync(0xffffffffu, w[i], lane);
        return r;
    }
};
template <> struct Raw<float> {
    float x[8];
    __device__ __forceinline__ void load(const float *p)
    {
        const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    }
    __device__ __forceinline__ void store(float *p) const
    {
        *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4 *>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0.f;
    }
    __device__ __forceinline__ void get(float (&y)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i];
    }
    __device__ __forceinline__ void get(uint64_t (&y)[4]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = pack2(x[2 * i], x[2 * i + 1]);
    }
    __device__ __forceinline__ void set(const float (&y)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = y[i];
    }
    __device__ __forceinline__ Raw from(int lane) const
    {
        Raw r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r.x[i] = __shfl_sync(0xffffffffu, x[i], lane);
        return r;
    }
};
__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// ---------------------------------------------------------------- single rows
// One row of a result by one warp, over exactly the places that its mask leaves.
// The tiled kernels multiply masked places by zero, which an infinity or a NaN in
// such a place turns into NaN; a row that comes out not finite is computed again
// here, where masked places are not read at all.  Lanes hold features lane + 32 u.
// A sum that is NaN stays so: a row stops there, as all do soon when everything is NaN.
// They count, so that a test can tell that nothing else sends rows here.
__device__ unsigned long long g_rows_again = 0;
__device__ __forceinline__ void count_row(int lane)
{
    if (lane == 0) atomicAdd(&g_rows_again, 1ull);
}

template <typename T>
struct RowArgs {
    Mask mask;
    Score score;
    Heads<const T> q, k, v, o, d_o;
    Heads<T> out, dq, dk, dv;
    float *lse;          // [n_q][T]
    const float *delta;  // [n_q][T], backward
    int n_q, n_kv, d;
};

template <typename T>
__device__ __forceinline__ void row_load(float (&x)[4], const T *p, int d, int lane)
{
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = lane + 32 * u < d ? load_f(p + lane + 32 * u) : 0.f;
}
// features [f0, f1) of a row
template <typename T>
__device__ __forceinline__ void row_store(T *p, const float (&x)[4], int f1, int lane, int f0 = 0)
{
#pragma unroll
    for (int u = 0; u < 4; ++u)
        if (lane + 32 * u >= f0 && lane + 32 * u < f1) store_f(p + lane + 32 * u, x[u]);
}
__device__ __forceinline__ float row_dot(const float (&a)[4], const float (&b)[4])
{
    return warp_sum(a[0] * b[0] + a[1] * b[1] + a[2] * b[2] + a[3] * b[3]);
}
// Whether all features of a row are NaN.
__device__ __forceinline__ bool all_nan(const float (&x)[4], int d, int lane)
{
    bool all = true;
#pragma unroll
    for (int u = 0; u < 4; ++u) all = all && (lane + 32 * u >= d || isnan(x[u]));
    return __all_sync(0xffffffffu, all);
}
// the score, and in `deriv` its derivative by scale q.k
__device__ __forceinline__ float row_score(const Score &s, float qk, int h, int i, int j, float *deriv)
{
    float x = qk * s.scale, g = 1.f;
    if (s.softcap > 0.f) {
        const float t = tanhf(x / s.softcap);
        x = s.softcap * t;
        g = 1.f - t * t;
    }
    if (s.slope) x -= s.slope[h] * fabsf((float)(i - j));
    if (deriv) *deriv = g;
    return x;
}

template <typename T>
__device__ __noinline__ void row_fwd(const RowArgs<T> &a, int i, int h, int lane)
{
    count_row(lane);
    const Range r = visible(a.mask, i);
    const int g = h / (a.n_q / a.n_kv);
    float q[4], acc[4] = {}, m = -INFINITY, l = 0.f;
    row_load(q, a.q.at(i, h), a.d, lane);
    for (int j = r.lo; j < r.hi; ++j) {
        float x[4];
        row_load(x, a.k.at(j, g), a.d, lane);
        const float s = row_score(a.score, row_dot(q, x), h, i, j, nullptr);
        row_load(x, a.v.at(j, g), a.d, lane);
        const float mn = fmaxf(m, s);
        const float c = m == -INFINITY ? 0.f : expf(m - mn), p = s == -INFINITY ? 0.f : expf(s - mn);
        m = mn, l = l * c + p;
#pragma unroll
        for (int u = 0; u < 4; ++u) acc[u] = acc[u] * c + p * x[u];
        if (isnan(l)) break;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int u = 0; u < 4; ++u) acc[u] *= inv;
    row_store(a.out.at(i, h), acc, a.d, lane);
    if (lane == 0) a.lse[(int64_t)h * a.mask.T + i] = l == 0.f ? -INFINITY : m + logf(l);
}

// p and ds of one pair
template <typename T>
__device__ __forceinline__ void row_pair(const RowArgs<T> &a, const float (&q)[4], const float (&k)[4], const float (&v)[4],
                                         const float (&d_o)[4], float lse, float delta, int h, int i, int j, float &p,
                                         float &ds)
{
    float g;
    p = expf(row_score(a.score, row_dot(q, k), h, i, j, &g) - lse);
    ds = p * (row_dot(d_o, v) - delta) * g * a.score.scale;
}

// features [f0, f1) of dq
template <typename T>
__device__ __noinline__ void row_dq(const RowArgs<T> &a, int i, int h, int lane, float delta, int f0, int f1)
{
    count_row(lane);
    const Range r = visible(a.mask, i);
    const int g = h / (a.n_q / a.n_kv);
    const float lse = a.lse[(int64_t)h * a.mask.T + i];
    float q[4], d_o[4], acc[4] = {};
    row_load(q, a.q.at(i, h), a.d, lane);
    row_load(d_o, a.d_o.at(i, h), a.d, lane);
    for (int j = r.lo; j < r.hi; ++j) {
        float k[4], v[4], p, ds;
        row_load(k, a.k.at(j, g), a.d, lane);
        row_load(v, a.v.at(j, g), a.d, lane);
        row_pair(a, q, k, v, d_o, lse, delta, h, i, j, p, ds);
#pragma unroll
        for (int u = 0; u < 4; ++u) acc[u] += ds * k[u];
        if (isnan(ds)) break;
    }
    row_store(a.dq.at(i, h), acc, min(f1, a.d), lane, f0);
}

// First query whose range ends after key j, and first whose range starts after it:
// the queries that see j are those from one to the other.
__device__ __forceinline__ Range seen_by(const Mask &m, int j)
{
    Range out;
    int a = -1, b = m.T;
    while (b - a > 1) {
        const int c = (a + b) >> 1;
        if (visible(m, c).hi > j) b = c;
        else a = c;
    }
    out.lo = b;
    a = b - 1, b = m.T;
    while (b - a > 1) {
        const int c = (a + b) >> 1;
        if (visible(m, c).lo > j) b = c;
        else a = c;
    }
    out.hi = b;
    return out;
}

template <typename T>
__device__ __noinline__ void row_dkv(const RowArgs<T> &a, int j, int g, int lane, bool to_dv, bool to_dk)
{
    count_row(lane);
    const Range r = seen_by(a.mask, j);
    const int group = a.n_q / a.n_kv;
    float k[4], v[4], dk[4] = {}, dv[4] = {};
    row_load(k, a.k.at(j, g), a.d, lane);
    row_load(v, a.v.at(j, g), a.d, lane);
    bool lost = false;
    for (int h = g * group; h < (g + 1) * group; ++h)
        for (int i = r.lo; i < r.hi && !lost; ++i) {
            float q[4], d_o[4], p, ds;
            row_load(q, a.q.at(i, h), a.d, lane);
            row_load(d_o, a.d_o.at(i, h), a.d, lane);
            row_pair(a, q, k, v, d_o, a.lse[(int64_t)h * a.mask.T + i], a.delta[(int64_t)h * a.mask.T + i], h, i, j, p, ds);
#pragma unroll
            for (int u = 0; u < 4; ++u) dk[u] += ds * q[u], dv[u] += p * d_o[u];
            lost = (!to_dk || isnan(ds)) && (!to_dv || all_nan(dv, a.d, lane));
        }
    if (to_dk) row_store(a.dk.at(j, g), dk, a.d, lane);
    if (to_dv) row_store(a.dv.at(j, g), dv, a.d, lane);
}

}  // namespace attn
}  // namespace noble
