// Norms of the queries and keys by head, their rotation by position, the gradients
// of both, and the same on the way into a paged cache.
//
// All of it moves every element once each way and is bound by that.  A lane holds 8
// consecutive features of a head (16 bytes of bf16), LP lanes a head, so a warp
// reads whole heads in 16-byte pieces; the sum of a norm is a butterfly over LP
// lanes.  A batch is kPasses * 32 / LP heads of one token and one kind (queries, keys or
// values), whose loads are all issued before the first is used; they stay packed, and it
// is the packed words that go to the other lane of a pair.  Gains are multiplied
// into the cosines and sines once per kind, which leaves two products and a scale
// per element.
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
    float eps, inv_d;
    int norm, interleaved;
    int lp, batches_q, batches_kv;  // lanes per head; batches of a token's queries, of its keys or values
    int take, groups;               // forward: batches of a warp, warps of a token
    uint32_t *status;
    // append
    const int64_t *slots;
    T *k_cache, *v_cache;
    int64_t capacity, page, row, head;
    int page_size;
};

using attn::Raw;
using attn::load8;

// Factors of a lane's 8 features: y_f = c x_f + s x_(other of f), s = 0 where f does not
// rotate; with gains (norm) c holds f's and s its partner's.
struct Turn {
    float c[8], s[8];
};
template <int MODE>
__device__ __forceinline__ int partner(int e, int rot, int interleaved)
{
    const int half = rot / 2;
    if (MODE == kInterleaved || (MODE == kAny && interleaved)) return e ^ 1;
    return e < half ? e + half : e - half;
}
// `row`: the token's row of the table; SIGN -1 turns back
template <int MODE, int SIGN>
__device__ __forceinline__ void load_turn(Turn &t, const float *row, int f, int rot, int interleaved)
{
    const int half = rot / 2;
#pragma unroll
    for (int i = 0; i < 8; ++i) t.c[i] = 1.f, t.s[i] = 0.f;
    if (MODE == kHalf) {
        if (f < rot) {
            const bool second = f >= half;
            load8(t.c, row + (second ? f - half : f));
            load8(t.s, row + half + (second ? f - half : f));
#pragma unroll
            for (int i = 0; i < 8; ++i) t.s[i] = (second ? SIGN : -SIGN) * t.s[i];
        }
    } else if (MODE == kInterleaved) {
        if (f < rot) {
            const float4 c = *reinterpret_cast<const float4 *>(row + f / 2), s = *reinterpret_cast<const float4 *>(row + half + f / 2);
            t.c[0] = t.c[1] = c.x, t.c[2] = t.c[3] = c.y, t.c[4] = t.c[5] = c.z, t.c[6] = t.c[7] = c.w;
            t.s[1] = SIGN * s.x, t.s[3] = SIGN * s.y, t.s[5] = SIGN * s.z, t.s[7] = SIGN * s.w;
            t.s[0] = -SIGN * s.x, t.s[2] = -SIGN * s.y, t.s[4] = -SIGN * s.z, t.s[6] = -SIGN * s.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = f + i;
            if (e < rot) {
                const int pair = interleaved ? e / 2 : e < half ? e : e - half;
                const bool first = interleaved ? e % 2 == 0 : e < half;
                t.c[i] = row[pair];
                t.s[i] = (first ? -SIGN : SIGN) * row[half + pair];
            }
        }
    }
}

// The other features of the pairs of a lane's 8.  `buf`: 256 floats of the warp (kAny).
template <int MODE, typename T>
__device__ __forceinline__ void others(float (&y)[8], const Raw<T> &r, const float (&x)[8], int f, int rot, int interleaved,
                                       float *buf, int lane)
{
    if (MODE == kHalf) {
        const int other = f >= rot ? lane : f < rot / 2 ? lane + rot / 16 : lane - rot / 16;
        r.from(other & 31).get(y);
    } else if (MODE == kInterleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i ^ 1];
    } else {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) buf[lane * 8 + i] = x[i];
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = f + i < rot ? buf[lane * 8 - f + partner<kAny>(f + i, rot, interleaved)] : 0.f;
    }
}
// x turned, in place; features that do not rotate do not meet their neighbours' values
template <int MODE>
__device__ __forceinline__ void turn8(float (&x)[8], const float (&y)[8], const Turn &t, int f, int rot)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = x[i] * t.c[i];
        x[i] = (MODE == kAny ? f + i < rot : f < rot) ? fmaf(y[i], t.s[i], a) : a;
    }
}

// LP: lanes of a head, 0 for a number that only the arguments know
template <int LP>
__device__ __forceinline__ float head_sum(float v, int lp)
{
#pragma unroll
    for (int o = 1; o < (LP ? LP : 32); o <<= 1) {
        const float w = __shfl_xor_sync(0xffffffffu, v, o);
        v += LP || o < lp ? w : 0.f;
    }
    return v;
}

// A warp: `take` batches of a token, the next one's loads in flight while one is worked on.
template <int MODE, bool APPEND, int LP, typename T>
__global__ void __launch_bounds__(32 * kWarps, sizeof(T) == 2 && MODE != kAny ? 3 : 2) fwd_kernel(const __grid_constant__ Args<T> a)
{
    __shared__ float bufs[MODE == kAny ? kWarps : 1][256];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int64_t u = (int64_t)blockIdx.x * kWarps + warp;
    if (u >= a.tokens * a.groups) return;
    // a 64-bit division costs as much as a head
    const int64_t t = a.groups == 1 ? u : u >> 32 ? u / a.groups : (uint32_t)u / (uint32_t)a.groups;
    const int lp = LP ? LP : a.lp, hp = 32 / lp, f = lane % lp * 8, own = lane / lp;
    const bool in = f < a.d;
    const int all = a.batches_q + (APPEND ? 2 : 1) * a.batches_kv;
    const int b0 = (int)(u - t * a.groups) * a.take, b1 = min(b0 + a.take, all);
    // batch b: heads first + own + p * hp of its kind (0 queries, 1 keys, 2 values)
    auto kind_of = [&](int b) { return b < a.batches_q ? 0 : b < a.batches_q + a.batches_kv ? 1 : 2; };
    auto first_of = [&](int b, int kind) { return (b - (kind ? a.batches_q + (kind - 1) * a.batches_kv : 0)) * kPasses * hp + own; };
    auto load = [&](Raw<T> (&r)[kPasses], int b) {
        const int kind = kind_of(b), h0 = first_of(b, kind), n = kind ? a.n_kv : a.n_q;
        const Heads<const T> &x = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            if (in && b < b1 && h0 + p * hp < n) r[p].load(x.at(t, h0 + p * hp) + f);
            else r[p].zero();
        }
    };
    Raw<T> r[kPasses];
    load(r, b0);
    const int pos = a.pos[t];
    const bool known = pos >= 0 && pos < a.positions;
    if (!known && lane == 0) raise_status(a.status, kStatusBadIndex);
    const float *row = a.table + (int64_t)(known ? pos : 0) * a.rot;
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
    Turn tn;
    int have = -1;  // the kind that tn is for
    for (int b = b0; b < b1; ++b) {
        const int kind = kind_of(b), h0 = first_of(b, kind), n = kind ? a.n_kv : a.n_q;
        Raw<T> next[kPasses];
        load(next, b + 1);
        if (APPEND && kind == 2) {
#pragma unroll
            for (int p = 0; p < kPasses; ++p)
                if (in && vc && h0 + p * hp < n) r[p].store(vc + (h0 + p * hp) * a.head + f);
        } else {
            const float *gain = kind ? a.gain_k : a.gain_q;
            if (kind != have) load_turn<MODE, 1>(tn, row, known && in ? f : a.rot, a.rot, a.interleaved);
            if (kind != have && gain && in) {
                float g[8];
                load8(g, gain + f);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    tn.c[i] *= g[i];
                    if (MODE == kInterleaved) tn.s[i] *= g[i ^ 1];
                    if (MODE == kAny && f + i < a.rot) tn.s[i] *= gain[partner<MODE>(f + i, a.rot, a.interleaved)];
                }
                if (MODE == kHalf && f < a.rot) {
                    load8(g, gain + partner<MODE>(f, a.rot, 0));
#pragma unroll
                    for (int i = 0; i < 8; ++i) tn.s[i] *= g[i];
                }
            }
            have = kind;
#pragma unroll
            for (int p = 0; p < kPasses; ++p) {
                const int h = h0 + p * hp;
                float x[8], y[8];
                r[p].get(x);
                others<MODE>(y, r[p], x, f, a.rot, a.interleaved, bufs[MODE == kAny ? warp : 0], lane);
                float scale = 1.f;
                if (a.norm) {
                    float s = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) s = fmaf(x[i], x[i], s);
                    scale = rsqrtf(fmaf(head_sum<LP>(s, a.lp), a.inv_d, a.eps));
                }
                turn8<MODE>(x, y, tn, f, a.rot);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = known ? x[i] * scale : 0.f;
                Raw<T> o;
                o.set(x);
                if (!in || h >= n) continue;
                if (kind == 0) o.store(a.q_out.at(t, h) + f);
                else if (!APPEND) o.store(a.k_out.at(t, h) + f);
                else if (kc) o.store(kc + h * a.head + f);
            }
        }
#pragma unroll
        for (int p = 0; p < kPasses; ++p) r[p] = next[p];
    }
}

// Persistent over the batches of the queries, then of the keys, so that a lane adds up its
// features' gain gradients in registers, the block in shared memory: one partial per block.
template <int MODE, int LP, typename T>
__global__ void __launch_bounds__(32 * kWarps, 2) bwd_kernel(const __grid_constant__ Args<T> a)
{
    __shared__ float bufs[kWarps][256];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int lp = LP ? LP : a.lp, hp = 32 / lp, f = lane % lp * 8, own = lane / lp;
    const bool in = f < a.d;
    for (int kind = 0; kind < 2; ++kind) {
        const Heads<const T> &xs = kind ? a.k : a.q, &ds = kind ? a.dk : a.dq;
        const Heads<T> &out = kind ? a.k_out : a.q_out;
        const float *gain = kind ? a.gain_k : a.gain_q;
        const int n = kind ? a.n_kv : a.n_q, per = kind ? a.batches_kv : a.batches_q;
        float g[8], sum[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = 1.f, sum[i] = 0.f;
        if (gain && in) load8(g, gain + f);
        // unit = (token, batch); a stride of the grid's warps is step_t tokens and step_b batches
        const int64_t u0 = (int64_t)blockIdx.x * kWarps + warp;
        const int stride = gridDim.x * kWarps, step_t = stride / per, step_b = stride - step_t * per;
        int64_t t = u0 / per;
        int b = (int)(u0 - t * per);
        int pos = t < a.tokens ? a.pos[t] : 0;
        while (t < a.tokens) {
            const int h0 = b * kPasses * hp + own;
            Raw<T> rx[kPasses], rd[kPasses];
#pragma unroll
            for (int p = 0; p < kPasses; ++p) {
                rx[p].zero(), rd[p].zero();
                if (in && h0 + p * hp < n) {
                    rd[p].load(ds.at(t, h0 + p * hp) + f);
                    if (a.norm) rx[p].load(xs.at(t, h0 + p * hp) + f);
                }
            }
            const bool known = pos >= 0 && pos < a.positions;
            if (!known && lane == 0) raise_status(a.status, kStatusBadIndex);
            Turn tn;
            load_turn<MODE, -1>(tn, a.table + (int64_t)(known ? pos : 0) * a.rot, known && in ? f : a.rot, a.rot, a.interleaved);
            int64_t t_next = t + step_t;
            b += step_b;
            if (b >= per) b -= per, ++t_next;
            if (t_next < a.tokens) pos = a.pos[t_next];
#pragma unroll
            for (int p = 0; p < kPasses; ++p) {
                const bool real = in && h0 + p * hp < n;
                float w[8], y[8];
                rd[p].get(w);
                others<MODE>(y, rd[p], w, f, a.rot, a.interleaved, bufs[warp], lane);
                turn8<MODE>(w, y, tn, f, a.rot);
                if (!known)
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = 0.f;
                if (a.norm) {
                    float x[8], s = 0.f;
                    rx[p].get(x);
#pragma unroll
                    for (int i = 0; i < 8; ++i) s = fmaf(x[i], x[i], s);
                    const float scale = rsqrtf(fmaf(head_sum<LP>(s, a.lp), a.inv_d, a.eps));
                    s = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        x[i] *= scale;
                        sum[i] = fmaf(w[i], x[i], sum[i]);  // 0 in lanes without a head
                        w[i] *= g[i];
                        s = fmaf(w[i], x[i], s);
                    }
                    s = head_sum<LP>(s, a.lp) * a.inv_d;
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = scale * fmaf(-x[i], s, w[i]);
                }
                Raw<T> o;
                o.set(w);
                if (real) o.store(out.at(t, h0 + p * hp) + f);
            }
            t = t_next;
        }
        if (!a.part) continue;
        // over the heads side by side in the warp, then over the warps, in order
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) bufs[warp][lane * 8 + i] = sum[i];
        __syncthreads();
        for (int e = threadIdx.x; e < a.d; e += 32 * kWarps) {
            float s = 0.f;
            for (int w = 0; w < kWarps; ++w)
                for (int j = 0; j < hp; ++j) s += bufs[w][j * lp * 8 + e];
            a.part[((int64_t)blockIdx.x * 2 + kind) * a.d + e] = s;
        }
        __syncthreads();
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
