// Attention on the CUDA cores, fp32 FMA throughout: the path of fp32 operands, and
// with NOBLE_ATTN_SIMT_ONLY of bf16 ones.  One pass over the keys with the running
// maximum and sum of a softmax (forward); probabilities again from lse (backward).
//
// Blocks of 32 x 64 scores, 128 threads of 4 x 4 each: small ones, so that several share an
// SM and hide each other's loads and barriers.  A step over four features
// takes 4 + 4 16-byte loads from shared memory for 64 FMAs a thread: rows padded by
// four floats make the strided loads of 16 consecutive rows free of conflicts.
// Backward in two kernels, one per side of the scores, so that every sum has one
// block and a fixed order: dk and dv by key block over the queries (and the query
// heads that share the key head), dq by query block over the keys.
//
// Bound by the reads from shared memory beside the FMAs, and by blocks of uneven length: 1024
// tokens, 16 heads of 64, causal, fp32: forward 125 us (17 TFLOP/s), backward 355 (15); both
// together 659 with blocks of 64 x 64.
#pragma once

#include "attn_mask.cuh"

namespace noble {
namespace attn {
namespace simt {

constexpr int kM = 32, kB = 64, kThreads = 128, kPP = kB + 4;  // rows and columns of a block

template <int DP> constexpr int kLd = DP + 4;  // floats of a padded row

// Rows [r0, r0 + ROWS) of head h as fp32, zeros at rows >= limit and features >= d.
template <int DP, int ROWS, typename T>
__device__ __forceinline__ void load_tile(float *sm, const Heads<const T> &x, int64_t h, int r0, int limit, int d)
{
#pragma unroll 8
    for (int c = threadIdx.x; c < ROWS * DP / 4; c += kThreads) {
        const int row = c / (DP / 4), f = c % (DP / 4) * 4;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r0 + row < limit && f < d) v = load4(x.at(r0 + row, h) + f);
        *reinterpret_cast<float4 *>(sm + row * kLd<DP> + f) = v;
    }
}

// s[r][c] = rows (ty + RS r) of A . rows (tx + 16 c) of B
template <int DP, int R = 4, int RS = 8>
__device__ __forceinline__ void dots(float (&s)[R][4], const float *A, const float *B, int ty, int tx)
{
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[r][c] = 0.f;
#pragma unroll 4
    for (int f = 0; f < DP; f += 4) {
        float4 a[R], b[4];
#pragma unroll
        for (int r = 0; r < R; ++r) a[r] = *reinterpret_cast<const float4 *>(A + (ty + RS * r) * kLd<DP> + f);
#pragma unroll
        for (int c = 0; c < 4; ++c) b[c] = *reinterpret_cast<const float4 *>(B + (tx + 16 * c) * kLd<DP> + f);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                s[r][c] = fmaf(a[r].x, b[c].x, s[r][c]);
                s[r][c] = fmaf(a[r].y, b[c].y, s[r][c]);
                s[r][c] = fmaf(a[r].z, b[c].z, s[r][c]);
                s[r][c] = fmaf(a[r].w, b[c].w, s[r][c]);
            }
    }
}

// acc[r][u] += sum_k P[ty + RS r][k] * B[k][features of thread tx]; features 64 u + 4 tx + 0..3
template <int DP, int R = 4, int RS = 8>
__device__ __forceinline__ void accumulate(float4 (&acc)[R][DP / 64], const float *P, const float *B, int ty, int tx)
{
#pragma unroll 2
    for (int k = 0; k < kB; k += 4) {
        float4 p[R];
#pragma unroll
        for (int r = 0; r < R; ++r) p[r] = *reinterpret_cast<const float4 *>(P + (ty + RS * r) * kPP + k);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int u = 0; u < DP / 64; ++u) {
                const float4 b = *reinterpret_cast<const float4 *>(B + (k + kk) * kLd<DP> + 64 * u + 4 * tx);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float w = kk == 0 ? p[r].x : kk == 1 ? p[r].y : kk == 2 ? p[r].z : p[r].w;
                    acc[r][u].x = fmaf(w, b.x, acc[r][u].x);
                    acc[r][u].y = fmaf(w, b.y, acc[r][u].y);
                    acc[r][u].z = fmaf(w, b.z, acc[r][u].z);
                    acc[r][u].w = fmaf(w, b.w, acc[r][u].w);
                }
            }
    }
}

template <int U>
__device__ __forceinline__ bool finite(const float4 (&x)[U])
{
    bool ok = true;
#pragma unroll
    for (int u = 0; u < U; ++u)
        ok = ok && isfinite(x[u].x) && isfinite(x[u].y) && isfinite(x[u].z) && isfinite(x[u].w);
    return ok;
}
template <typename T, int U>
__device__ __forceinline__ void store_row(T *p, const float4 (&x)[U], float f, int d, int tx)
{
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (64 * u + 4 * tx < d)
            store4(p + 64 * u + 4 * tx, make_float4(x[u].x * f, x[u].y * f, x[u].z * f, x[u].w * f));
}

// shared memory, floats
template <int DP> constexpr int kFwdFloats = (kM + kB) * kLd<DP> + kM * kPP;
template <int DP> constexpr int kBwdFloats = 2 * (kM + kB) * kLd<DP> + 2 * kM * kPP;

// s in place of q.k, with its derivative by scale q.k (softcap only)
__device__ __forceinline__ float score(const Score &sc, float slope, float qk, int far, float *deriv)
{
    float x = qk * sc.scale;
    if (sc.softcap > 0.f) {
        const float t = tanhf(x / sc.softcap);
        if (deriv) *deriv = 1.f - t * t;
        x = sc.softcap * t;
    }
    return x - slope * fabsf((float)far);
}

// grid: x = query blocks (the last, with the most keys under a causal mask, first), y = query heads
template <int DP, typename T>
__global__ void __launch_bounds__(kThreads) fwd_kernel(const __grid_constant__ RowArgs<T> a)
{
    extern __shared__ float sm[];
    float *Q = sm, *KV = Q + kM * kLd<DP>, *P = KV + kB * kLd<DP>;
    __shared__ int redo[kM];
    const int T_ = a.mask.T, tid = threadIdx.x, tx = tid % 16, ty = tid / 16;
    const int i0 = (int)(gridDim.x - 1 - blockIdx.x) * kM, h = blockIdx.y, g = h / (a.n_q / a.n_kv);
    const float slope = a.score.slope ? a.score.slope[h] : 0.f;
    Range rg[4];
    float m[4], l[4];
    float4 acc[4][DP / 64];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int i = i0 + ty + 8 * r;
        rg[r] = i < T_ ? visible(a.mask, i) : Range{0, 0};
        m[r] = -INFINITY, l[r] = 0.f;
#pragma unroll
        for (int u = 0; u < DP / 64; ++u) acc[r][u] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    const int lo = visible(a.mask, i0).lo, hi = visible(a.mask, min(i0 + kM, T_) - 1).hi;
    load_tile<DP, kM>(Q, a.q, h, i0, T_, a.d);
    for (int j0 = lo; j0 < hi; j0 += kB) {
        __syncthreads();
        load_tile<DP, kB>(KV, a.k, g, j0, hi, a.d);
        __syncthreads();
        float s[4][4];
        dots<DP>(s, Q, KV, ty, tx);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = i0 + ty + 8 * r;
            float top = m[r];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int j = j0 + tx + 16 * c;
                s[r][c] = j >= rg[r].lo && j < rg[r].hi ? score(a.score, slope, s[r][c], i - j, nullptr) : -INFINITY;
                top = fmaxf(top, s[r][c]);
            }
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            const float base = top == -INFINITY ? 0.f : top;
            float sum = 0.f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                s[r][c] = exp2f((s[r][c] - base) * kLog2e);
                sum += s[r][c];
                P[(ty + 8 * r) * kPP + tx + 16 * c] = s[r][c];
            }
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            const float f = exp2f((m[r] - base) * kLog2e);
            m[r] = top, l[r] = l[r] * f + sum;
#pragma unroll
            for (int u = 0; u < DP / 64; ++u)
                acc[r][u].x *= f, acc[r][u].y *= f, acc[r][u].z *= f, acc[r][u].w *= f;
        }
        __syncthreads();
        load_tile<DP, kB>(KV, a.v, g, j0, hi, a.d);
        __syncthreads();
        accumulate<DP>(acc, P, KV, ty, tx);
    }
    if (tid < kM) redo[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int i = i0 + ty + 8 * r;
        if (i >= T_) continue;
        const bool none = rg[r].lo >= rg[r].hi;
        if (none)
#pragma unroll
            for (int u = 0; u < DP / 64; ++u) acc[r][u] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (!finite(acc[r]) || !isfinite(none ? 0.f : l[r])) redo[ty + 8 * r] = 1;
        store_row(a.out.at(i, h), acc[r], l[r] > 0.f ? 1.f / l[r] : 0.f, a.d, tx);
        if (tx == 0) a.lse[(int64_t)h * T_ + i] = l[r] > 0.f ? m[r] + logf(l[r]) : -INFINITY;
    }
    __syncthreads();
    for (int r = tid / 32; r < kM; r += kThreads / 32)
        if (redo[r]) row_fwd(a, i0 + r, h, tid % 32);
}

// delta[h][i] = sum_f o do; with ranges, also the range of every token.  Bound by reading o
// and do: a lane takes 8 features of each, LP lanes a head, and four heads at a time
// (grid strides apart) are in flight.  16384 tokens, 16 heads of 128: 24 us, 5.6 TB/s.
template <typename T, int LP>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 4 : 2) delta_kernel(const __grid_constant__ RowArgs<T> a, float *delta, int2 *ranges, int step_t,
                                                    int step_h)
{
    // head u = (t, h) of all; a step of the grid is step_t tokens and step_h heads
    constexpr int kAtOnce = 4, kPer = 256 / LP;
    const int f = threadIdx.x % LP * 8;
    const int64_t u = (int64_t)blockIdx.x * kPer + threadIdx.x / LP;
    int t = (int)(u / a.n_q), h = (int)(u % a.n_q);
    const int steps = (int)(((int64_t)a.mask.T * a.n_q - (int64_t)blockIdx.x * kPer + (int64_t)gridDim.x * kPer - 1) / ((int64_t)gridDim.x * kPer));
    for (int k = 0; k < steps; k += kAtOnce) {
        Raw<T> x[kAtOnce], y[kAtOnce];
        int ts[kAtOnce], hs[kAtOnce];
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) {
            ts[e] = t, hs[e] = h;
            t += step_t, h += step_h;
            if (h >= a.n_q) h -= a.n_q, ++t;
            const bool in = ts[e] < a.mask.T && f < a.d;
            x[e].zero(), y[e].zero();
            if (in) x[e].load(a.o.at(ts[e], hs[e]) + f), y[e].load(a.d_o.at(ts[e], hs[e]) + f);
        }
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) {
            float s = 0.f, v[8], w[8];
            x[e].get(v), y[e].get(w);
#pragma unroll
            for (int c = 0; c < 8; ++c) s = fmaf(v[c], w[c], s);
#pragma unroll
            for (int o = 1; o < LP; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (ts[e] < a.mask.T && f == 0) {
                delta[(int64_t)hs[e] * a.mask.T + ts[e]] = s;
                if (ranges && hs[e] == 0) {
                    const Range r = visible(a.mask, ts[e]);
                    ranges[ts[e]] = make_int2(r.lo, r.hi);
                }
            }
        }
    }
}

// First query of the block of queries that sees anything of keys [j0, j1), and one
// past the last: by the ranges' order.
__device__ __forceinline__ Range queries_of(const int2 *ranges, int T, int j0, int j1)
{
    Range out;
    int a = -1, b = T;
    while (b - a > 1) {
        const int c = (a + b) >> 1;
        if (ranges[c].y > j0) b = c;
        else a = c;
    }
    out.lo = b;
    a = b - 1, b = T;
    while (b - a > 1) {
        const int c = (a + b) >> 1;
        if (ranges[c].x >= j1) b = c;
        else a = c;
    }
    out.hi = b;
    return out;
}

// grid: x = key blocks, y = key heads.  Rows of the score block are keys.
template <int DP, typename T>
__global__ void __launch_bounds__(kThreads) dkv_kernel(const __grid_constant__ RowArgs<T> a, const int2 *ranges)
{
    extern __shared__ float sm[];
    float *K = sm, *V = K + kM * kLd<DP>, *Q = V + kM * kLd<DP>, *DO = Q + kB * kLd<DP>;
    float *P = DO + kB * kLd<DP>, *DS = P + kM * kPP;
    __shared__ int redo[kM];
    __shared__ int2 rg[kB];
    __shared__ float lse[kB], delta[kB];
    const int T_ = a.mask.T, tid = threadIdx.x, tx = tid % 16, ty = tid / 16;
    const int j0 = blockIdx.x * kM, g = blockIdx.y, group = a.n_q / a.n_kv;
    const Range qs = queries_of(ranges, T_, j0, min(j0 + kM, docs_end(a.mask)));
    float4 dk[4][DP / 64], dv[4][DP / 64];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int u = 0; u < DP / 64; ++u) dk[r][u] = dv[r][u] = make_float4(0.f, 0.f, 0.f, 0.f);
    load_tile<DP, kM>(K, a.k, g, j0, T_, a.d);
    load_tile<DP, kM>(V, a.v, g, j0, T_, a.d);
    for (int h = g * group; h < (g + 1) * group; ++h) {
        const float slope = a.score.slope ? a.score.slope[h] : 0.f;
        for (int i0 = qs.lo; i0 < qs.hi; i0 += kB) {
            __syncthreads();
            load_tile<DP, kB>(Q, a.q, h, i0, qs.hi, a.d);
            load_tile<DP, kB>(DO, a.d_o, h, i0, qs.hi, a.d);
            if (tid < kB) {
                const int i = i0 + tid;
                rg[tid] = i < qs.hi ? ranges[i] : make_int2(0, 0);
                lse[tid] = i < qs.hi ? a.lse[(int64_t)h * T_ + i] : 0.f;
                delta[tid] = i < qs.hi ? a.delta[(int64_t)h * T_ + i] : 0.f;
            }
            __syncthreads();
            float s[4][4], dp[4][4];
            dots<DP>(s, K, Q, ty, tx);
            dots<DP>(dp, V, DO, ty, tx);
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int j = j0 + ty + 8 * r, q = tx + 16 * c;
                    float p = 0.f, ds = 0.f;
                    if (j >= rg[q].x && j < rg[q].y) {
                        float g1 = 1.f;
                        const float x = score(a.score, slope, s[r][c], i0 + q - j, &g1);
                        p = exp2f((x - lse[q]) * kLog2e);
                        ds = p * (dp[r][c] - delta[q]) * g1;
                    }
                    P[(ty + 8 * r) * kPP + q] = p;
                    DS[(ty + 8 * r) * kPP + q] = ds;
                }
            __syncthreads();
            accumulate<DP>(dv, P, DO, ty, tx);
            accumulate<DP>(dk, DS, Q, ty, tx);
        }
    }
    if (tid < kM) redo[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int j = j0 + ty + 8 * r;
        if (j >= T_) continue;
        if (!finite(dk[r]) || !finite(dv[r])) redo[ty + 8 * r] = 1;
        store_row(a.dk.at(j, g), dk[r], a.score.scale, a.d, tx);
        store_row(a.dv.at(j, g), dv[r], 1.f, a.d, tx);
    }
    __syncthreads();
    for (int r = tid / 32; r < kM; r += kThreads / 32)
        if (redo[r]) row_dkv(a, j0 + r, g, tid % 32, true, true);
}

// grid as fwd_kernel's.  Where one block of keys is all that the queries see, delta is
// summed from p and dp themselves and replaces the one of the rounded o in `delta_out`:
// with few keys, dp - delta can be as small as that rounding.  Runs before dkv_kernel.
template <int DP, typename T>
__global__ void __launch_bounds__(kThreads) dq_kernel(const __grid_constant__ RowArgs<T> a, float *delta_out)
{
    extern __shared__ float sm[];
    float *Q = sm, *DO = Q + kM * kLd<DP>, *K = DO + kM * kLd<DP>, *V = K + kB * kLd<DP>, *DS = V + kB * kLd<DP>;
    __shared__ int redo[kM];
    const int T_ = a.mask.T, tid = threadIdx.x, tx = tid % 16, ty = tid / 16;
    const int i0 = (int)(gridDim.x - 1 - blockIdx.x) * kM, h = blockIdx.y, g = h / (a.n_q / a.n_kv);
    const float slope = a.score.slope ? a.score.slope[h] : 0.f;
    Range rg[4];
    float lse[4], delta[4];
    float4 dq[4][DP / 64];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int i = i0 + ty + 8 * r;
        rg[r] = i < T_ ? visible(a.mask, i) : Range{0, 0};
        lse[r] = i < T_ ? a.lse[(int64_t)h * T_ + i] : 0.f;
        delta[r] = i < T_ ? a.delta[(int64_t)h * T_ + i] : 0.f;
#pragma unroll
        for (int u = 0; u < DP / 64; ++u) dq[r][u] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    const int lo = visible(a.mask, i0).lo, hi = visible(a.mask, min(i0 + kM, T_) - 1).hi;
    const bool one = hi - lo <= kB;
    load_tile<DP, kM>(Q, a.q, h, i0, T_, a.d);
    load_tile<DP, kM>(DO, a.d_o, h, i0, T_, a.d);
    for (int j0 = lo; j0 < hi; j0 += kB) {
        __syncthreads();
        load_tile<DP, kB>(K, a.k, g, j0, hi, a.d);
        load_tile<DP, kB>(V, a.v, g, j0, hi, a.d);
        __syncthreads();
        float s[4][4], dp[4][4];
        dots<DP>(s, Q, K, ty, tx);
        dots<DP>(dp, DO, V, ty, tx);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float g1[4], sum = 0.f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int j = j0 + tx + 16 * c;
                g1[c] = 1.f;
                const bool in = j >= rg[r].lo && j < rg[r].hi;
                const float x = in ? score(a.score, slope, s[r][c], i0 + ty + 8 * r - j, &g1[c]) : 0.f;
                s[r][c] = in ? exp2f((x - lse[r]) * kLog2e) : 0.f;
                if (!in) dp[r][c] = 0.f;
                sum = fmaf(s[r][c], dp[r][c], sum);
            }
            if (one) {
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                delta[r] = sum;
                if (tx == 0 && rg[r].lo < rg[r].hi) delta_out[(int64_t)h * T_ + i0 + ty + 8 * r] = sum;
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int j = j0 + tx + 16 * c;
                DS[(ty + 8 * r) * kPP + tx + 16 * c] =
                    j >= rg[r].lo && j < rg[r].hi ? s[r][c] * (dp[r][c] - delta[r]) * g1[c] : 0.f;
            }
        }
        __syncthreads();
        accumulate<DP>(dq, DS, K, ty, tx);
    }
    if (tid < kM) redo[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int i = i0 + ty + 8 * r;
        if (i >= T_) continue;
        if (rg[r].lo >= rg[r].hi)
#pragma unroll
            for (int u = 0; u < DP / 64; ++u) dq[r][u] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (!finite(dq[r])) redo[ty + 8 * r] = 1;
        store_row(a.dq.at(i, h), dq[r], a.score.scale, a.d, tx);
    }
    __syncthreads();
    for (int r = tid / 32; r < kM; r += kThreads / 32)
        if (redo[r]) row_dq(a, i0 + r, h, tid % 32, delta_out[(int64_t)h * T_ + i0 + r], 0, a.d);
}

}  // namespace simt
}  // namespace attn
}  // namespace noble
