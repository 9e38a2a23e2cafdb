// Norms of the queries and keys by head, their rotation by position, the gradients
// of both, and the same on the way into a paged cache.
//
// All of it moves every element once each way and is bound by that.  A lane holds 8
// consecutive features of a head (16 bytes of bf16), LP lanes a head, so a warp
// reads whole heads in 16-byte pieces; the sum of a norm is a butterfly over LP
// lanes.  A warp takes kPasses * 32 / LP heads of one token at a time, whose loads are
// all issued before the first is used and which share the token's cosines and sines.
#pragma once

#include "attn_mask.cuh"

namespace noble {
namespace rope {

using attn::Heads;

// How a lane finds the other feature of a pair:
enum : int {
    kHalf = 0,         // (i, i + rot/2), rot/2 a multiple of 8: the same place of another lane
    kInterleaved = 1,  // (2i, 2i+1), rot a multiple of 8: in the lane
    kAny = 2,          // either layout at any size: through shared memory
};
constexpr int kPasses = 4, kWarps = 8;

template <typename T>
struct Args {
    Heads<const T> q, k, v, dq, dk;
    Heads<T> q_out, k_out;
    const int32_t *pos;
    const float *table, *gain_q, *gain_k;  // gains NULL: ones
    float *part;                           // [blocks][2][d]: partial gain gradients, or NULL
    int64_t tokens;
    int n_q, n_kv, d, rot, positions;
    float eps;
    int norm, interleaved;
    int lp, per_token;  // lanes per head; units of heads per token
    uint32_t *status;
    // append
    const int64_t *slots;
    T *k_cache, *v_cache;
    int64_t capacity, page, row, head;
    int page_size;
};

__device__ __forceinline__ void load8(float (&x)[8], const float *p)
{
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
__device__ __forceinline__ void load8(float (&x)[8], const __nv_bfloat16 *p)
{
    const uint4 u = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&w[i]));
        x[2 * i] = f.x, x[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ void store8(float *p, const float (&x)[8])
{
    *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float (&x)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<uint32_t *>(&b);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// Cosines and signed sines of a lane's 8 features: y_f = c x_f + s x_(other of f).
struct Turn {
    float c[8], s[8];
};
template <int MODE>
__device__ __forceinline__ void load_turn(Turn &t, const float *row, int f, int rot, int interleaved)
{
    const int half = rot / 2;
    if (MODE == kHalf) {
        if (f < rot) {
            const bool second = f >= half;
            load8(t.c, row + (second ? f - half : f));
            load8(t.s, row + half + (second ? f - half : f));
            if (!second)
#pragma unroll
                for (int i = 0; i < 8; ++i) t.s[i] = -t.s[i];
            return;
        }
    } else if (MODE == kInterleaved) {
        if (f < rot) {
            const float4 c = *reinterpret_cast<const float4 *>(row + f / 2), s = *reinterpret_cast<const float4 *>(row + half + f / 2);
            t.c[0] = t.c[1] = c.x, t.c[2] = t.c[3] = c.y, t.c[4] = t.c[5] = c.z, t.c[6] = t.c[7] = c.w;
            t.s[1] = s.x, t.s[3] = s.y, t.s[5] = s.z, t.s[7] = s.w;
            t.s[0] = -s.x, t.s[2] = -s.y, t.s[4] = -s.z, t.s[6] = -s.w;
            return;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = f + i;
            t.c[i] = 1.f, t.s[i] = 0.f;
            if (e < rot) {
                const int pair = interleaved ? e / 2 : e < half ? e : e - half;
                const bool first = interleaved ? e % 2 == 0 : e < half;
                t.c[i] = row[pair];
                t.s[i] = first ? -row[half + pair] : row[half + pair];
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) t.c[i] = 1.f, t.s[i] = 0.f;
}

// Rotates by the angle, or back (SIGN -1).  `buf`: 256 floats of the warp (kAny).
template <int MODE, int SIGN>
__device__ __forceinline__ void turn8(float (&x)[8], const Turn &t, int f, int rot, int interleaved, float *buf, int lane)
{
    float y[8];
    const int half = rot / 2;
    if (MODE == kHalf) {
        // lanes of features past `rot` multiply what they get by 0 unless it is not finite: they keep theirs
        const int other = f < half ? lane + half / 8 : lane - half / 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __shfl_sync(0xffffffffu, x[i], other & 31);
    } else if (MODE == kInterleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i ^ 1];
    } else {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) buf[lane * 8 + i] = x[i];
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = f + i, o = interleaved ? e ^ 1 : e < half ? e + half : e - half;
            y[i] = e < rot ? buf[lane * 8 - f + o] : 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (MODE == kAny ? f + i < rot : f < rot) x[i] = x[i] * t.c[i] + (SIGN > 0 ? y[i] : -y[i]) * t.s[i];
}

__device__ __forceinline__ float head_sum(float v, int lp)
{
    for (int o = 1; o < lp; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// One unit: heads [first, first + kPasses * 32 / lp) of a token.
template <int MODE, bool APPEND, typename T>
__global__ void __launch_bounds__(32 * kWarps) fwd_kernel(const __grid_constant__ Args<T> a)
{
    __shared__ float bufs[MODE == kAny ? kWarps : 1][256];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int64_t u = (int64_t)blockIdx.x * kWarps + warp;
    if (u >= a.tokens * a.per_token) return;
    const int64_t t = u / a.per_token;
    const int hp = 32 / a.lp, f = lane % a.lp * 8;
    const int first = (int)(u % a.per_token) * kPasses * hp + lane / a.lp;
    const int heads = a.n_q + a.n_kv + (APPEND ? a.n_kv : 0);
    const bool in = f < a.d;
    float x[kPasses][8];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const int h = first + p * hp;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[p][i] = 0.f;
        if (in && h < heads)
            load8(x[p], (h < a.n_q                        ? a.q.at(t, h)
                         : !APPEND || h < a.n_q + a.n_kv ? a.k.at(t, h - a.n_q)
                                                          : a.v.at(t, h - a.n_q - a.n_kv)) + f);
    }
    const int pos = a.pos[t];
    const bool known = pos >= 0 && pos < a.positions;
    if (!known && lane == 0) raise_status(a.status, kStatusBadIndex);
    Turn tn;
    load_turn<MODE>(tn, a.table + (int64_t)(known ? pos : 0) * a.rot, in ? f : a.rot, a.rot, a.interleaved);
    float gq[8], gk[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) gq[i] = gk[i] = 1.f;
    if (in && a.gain_q) load8(gq, a.gain_q + f);
    if (in && a.gain_k) load8(gk, a.gain_k + f);
    T *kc = nullptr, *vc = nullptr;
    if (APPEND) {
        const int64_t slot = a.slots[t];
        if (slot >= a.capacity) {
            if (lane == 0) raise_status(a.status, kStatusBadIndex);
        } else if (slot >= 0) {
            const int64_t at = slot / a.page_size * a.page + slot % a.page_size * a.row;
            kc = a.k_cache + at, vc = a.v_cache + at;
        }
    }
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const int h = first + p * hp;
        const bool is_q = h < a.n_q, is_v = APPEND && h >= a.n_q + a.n_kv;
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = x[p][i];
        if (a.norm) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s = fmaf(w[i], w[i], s);
            const float r = 1.f / sqrtf(head_sum(s, a.lp) / (float)a.d + a.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] *= r * (is_q ? gq[i] : gk[i]);
        }
        turn8<MODE, 1>(w, tn, f, a.rot, a.interleaved, bufs[MODE == kAny ? warp : 0], lane);
        if (!known)
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = 0.f;
        if (!in || h >= heads) continue;
        if (is_q) store8(a.q_out.at(t, h) + f, w);
        else if (!APPEND) store8(a.k_out.at(t, h - a.n_q) + f, w);
        else if (!is_v && kc) store8(kc + (h - a.n_q) * a.head + f, w);
        else if (is_v && vc) store8(vc + (h - a.n_q - a.n_kv) * a.head + f, x[p]);
    }
}

// Persistent over units, so that a lane adds up its features' gain gradients in
// registers, the block in shared memory; one partial per block.
template <int MODE, typename T>
__global__ void __launch_bounds__(32 * kWarps) bwd_kernel(const __grid_constant__ Args<T> a)
{
    constexpr int kP = 2;  // passes in flight: x and dy of each
    __shared__ float bufs[kWarps][256];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int hp = 32 / a.lp, f = lane % a.lp * 8;
    const int heads = a.n_q + a.n_kv;
    const bool in = f < a.d;
    float gq[8], gk[8], sq[8], sk[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) gq[i] = gk[i] = 1.f, sq[i] = sk[i] = 0.f;
    if (in && a.gain_q) load8(gq, a.gain_q + f);
    if (in && a.gain_k) load8(gk, a.gain_k + f);
    for (int64_t u = (int64_t)blockIdx.x * kWarps + warp; u < a.tokens * a.per_token; u += (int64_t)gridDim.x * kWarps) {
        const int64_t t = u / a.per_token;
        const int pos = a.pos[t];
        const bool known = pos >= 0 && pos < a.positions;
        if (!known && lane == 0) raise_status(a.status, kStatusBadIndex);
        Turn tn;
        load_turn<MODE>(tn, a.table + (int64_t)(known ? pos : 0) * a.rot, in ? f : a.rot, a.rot, a.interleaved);
#pragma unroll 1
        for (int p0 = 0; p0 < kPasses; p0 += kP) {
            float x[kP][8], w[kP][8];
#pragma unroll
            for (int p = 0; p < kP; ++p) {
                const int h = (int)(u % a.per_token) * kPasses * hp + lane / a.lp + (p0 + p) * hp;
#pragma unroll
                for (int i = 0; i < 8; ++i) x[p][i] = w[p][i] = 0.f;
                if (in && h < heads) {
                    load8(w[p], (h < a.n_q ? a.dq.at(t, h) : a.dk.at(t, h - a.n_q)) + f);
                    if (a.norm) load8(x[p], (h < a.n_q ? a.q.at(t, h) : a.k.at(t, h - a.n_q)) + f);
                }
            }
#pragma unroll
            for (int p = 0; p < kP; ++p) {
                const int h = (int)(u % a.per_token) * kPasses * hp + lane / a.lp + (p0 + p) * hp;
                const bool is_q = h < a.n_q, real = in && h < heads;
                turn8<MODE, -1>(w[p], tn, f, a.rot, a.interleaved, bufs[warp], lane);
                if (!known)
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[p][i] = 0.f;
                if (a.norm) {
                    float s = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) s = fmaf(x[p][i], x[p][i], s);
                    const float r = 1.f / sqrtf(head_sum(s, a.lp) / (float)a.d + a.eps);
                    s = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        x[p][i] *= r;
                        const float g = w[p][i] * x[p][i];
                        if (real && is_q) sq[i] += g;
                        if (real && !is_q) sk[i] += g;
                        w[p][i] *= is_q ? gq[i] : gk[i];
                        s = fmaf(w[p][i], x[p][i], s);
                    }
                    s = head_sum(s, a.lp) / (float)a.d;
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[p][i] = r * (w[p][i] - x[p][i] * s);
                }
                if (!real) continue;
                if (is_q) store8(a.q_out.at(t, h) + f, w[p]);
                else store8(a.k_out.at(t, h - a.n_q) + f, w[p]);
            }
        }
    }
    if (!a.part) return;
    // over the heads side by side in the warp, then over the warps, in order
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) bufs[warp][lane * 8 + i] = which ? sk[i] : sq[i];
        __syncthreads();
        for (int e = threadIdx.x; e < a.d; e += 32 * kWarps) {
            float s = 0.f;
            for (int w = 0; w < kWarps; ++w)
                for (int g = 0; g < hp; ++g) s += bufs[w][g * a.lp * 8 + e];
            a.part[((int64_t)blockIdx.x * 2 + which) * a.d + e] = s;
        }
    }
}

// dgain[which][e] = sum of the blocks' partials: a warp per output, its lanes over
// blocks lane, lane + 32, ... in order, then a butterfly
__global__ void __launch_bounds__(256) gain_kernel(const float *part, int blocks, int d, float *dgain_q, float *dgain_k)
{
    const int e = blockIdx.x * 8 + threadIdx.x / 32, lane = threadIdx.x % 32;
    if (e >= 2 * d) return;
    float s = 0.f;
    for (int b = lane; b < blocks; b += 32) s += part[(int64_t)b * 2 * d + e];
    s = attn::warp_sum(s);
    float *out = e < d ? dgain_q : dgain_k;
    if (lane == 0 && out) out[e % d] = s;
}

struct TableArgs {
    double log2_base, factor, original, low, high, amplitude;
    int64_t positions;
    int rot;
};
__global__ void __launch_bounds__(256) table_kernel(const TableArgs a, float *table)
{
    const int half = a.rot / 2;
    const int64_t n = a.positions * half;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (int64_t)gridDim.x * 256) {
        const int64_t p = e / half;
        const int i = (int)(e % half);
        double f = exp2(-2.0 * i / a.rot * a.log2_base);
        if (a.factor != 1.0) {
            const double turns = a.original * f / 6.283185307179586476925;
            const double g = turns >= a.high ? 1.0 : turns <= a.low ? 0.0 : (turns - a.low) / (a.high - a.low);
            f *= g + (1.0 - g) / a.factor;
        }
        double s, c;
        sincos((double)p * f, &s, &c);
        table[p * a.rot + i] = (float)(a.amplitude * c);
        table[p * a.rot + half + i] = (float)(a.amplitude * s);
    }
}

}  // namespace rope
}  // namespace noble
