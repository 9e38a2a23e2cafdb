// Norms of the queries and keys by head, their rotation by position, the gradients
// of both, and the same on the way into a paged cache.
//
// All of it moves every element once each way and is bound by that.  A lane holds 8
// consecutive features of a head (16 bytes of bf16), LP lanes a head, so a warp
// reads whole heads in 16-byte pieces; the sums of norms go over LP
// lanes.  A batch is kPasses * 32 / LP heads of one token and one kind (queries, keys or
// values), copied to shared memory by the lanes that will use it; the values stay packed until
// then, and it is the packed words that go to the other lane of a pair.  Arithmetic is two
// features per instruction.  Gains are multiplied
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
using attn::fma2;
using attn::load8;
using attn::mul2;
using attn::pack2;
using attn::sum2;
using attn::unpack2;

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

// The other features of the pairs of a lane's 8, zeros for those that do not rotate (which
// so do not meet their neighbours' values).  `buf`: 256 floats of the warp (kAny).
template <int MODE, typename T>
__device__ __forceinline__ void others(uint64_t (&y)[4], const Raw<T> &r, int f, int rot, int interleaved, float *buf, int lane)
{
    if (MODE == kHalf) {
        Raw<T> o = r.from((f >= rot ? lane : f < rot / 2 ? lane + rot / 16 : lane - rot / 16) & 31);
        if (f >= rot) o.zero();
        o.get(y);
    } else if (MODE == kInterleaved) {
        Raw<T> o = r;
        if (f >= rot) o.zero();
        float x[8];
        o.get(x);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = pack2(x[2 * i + 1], x[2 * i]);
    } else {
        float x[8];
        r.get(x);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) buf[lane * 8 + i] = x[i];
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = f + i < rot ? buf[lane * 8 - f + partner<kAny>(f + i, rot, interleaved)] : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = pack2(x[2 * i], x[2 * i + 1]);
    }
}
__device__ __forceinline__ void pack8(uint64_t (&p)[4], const float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = pack2(x[2 * i], x[2 * i + 1]);
}

// v[i] = the sum of every v[i] over the head's LP lanes (LP 0: lp of them, which only the
// arguments know).  At each step of the butterfly a lane keeps half of the values, while there are
// several, and hands the other half on; the sums go back to all at the end: 16 exchanges
// for 8 values and 16 lanes, where a butterfly each would take 32, at one per clock and SM.
template <int LP, int N>
__device__ __forceinline__ void head_sums(float (&v)[N], int lp, int lane)
{
    if constexpr (LP == 0) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float w = __shfl_xor_sync(0xffffffffu, v[i], o);
                v[i] += o < lp ? w : 0.f;
            }
    } else {
        static_assert(LP >= N, "lanes for all values");
        float u[N];
#pragma unroll
        for (int i = 0; i < N; ++i) u[i] = v[i];
#pragma unroll
        for (int o = 1; o < LP; o <<= 1) {
            const int n = N / (2 * o);  // values that are kept: those with this lane's bits so far
            if (n) {
#pragma unroll
                for (int i = 0; i < n; ++i) {
                    const float give = lane & o ? u[i] : u[i + n];
                    u[i] = (lane & o ? u[i + n] : u[i]) + __shfl_xor_sync(0xffffffffu, give, o);
                }
            } else {
                u[0] += __shfl_xor_sync(0xffffffffu, u[0], o);
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            int from = 0;  // bit by bit, the upper half of what was left came from lanes with the bit set
            for (int o = 1, n = N / 2, at = i; n; o <<= 1, n >>= 1)
                if (at >= n) from |= o, at -= n;
            v[i] = __shfl_sync(0xffffffffu, u[0], (lane & ~(LP - 1)) | from);
        }
    }
}

// 16 bytes to shared memory, zeros if they are not `real`; a lane waits for its own.
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool real)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }
// What a lane copied: pieces of 16 bytes, 512 apart.
template <typename T>
__device__ __forceinline__ void taken(Raw<T> &r, const char *at)
{
#pragma unroll
    for (int c = 0; c < (int)sizeof(T) / 2; ++c) reinterpret_cast<uint4 *>(&r)[c] = *reinterpret_cast<const uint4 *>(at + c * 512);
}

// A warp: `take` batches of a token, which wait in shared memory: what is on its way costs no
// registers there.  Bound by reading and
// writing with the latency of what comes first (position, then its cosines): 16384 tokens of
// 16 + 16 heads of 128 features 57 us, 4.7 TB/s (a batch ahead in registers 63); fp32 118, 4.6.
template <typename T> constexpr int kFwdRing = sizeof(T) == 2 ? 4 : 3;    // batches
template <typename T> constexpr int kFwdBlocks = sizeof(T) == 2 ? 3 : 2;  // of an SM
template <typename T> constexpr uint32_t kFwdBytes = kWarps * kFwdRing<T> * kPasses * 256 * sizeof(T);
template <int MODE, bool APPEND, int LP, typename T>
__global__ void __launch_bounds__(32 * kWarps, MODE == kAny ? 2 : kFwdBlocks<T>) fwd_kernel(const __grid_constant__ Args<T> a)
{
    extern __shared__ __align__(16) char ring[];  // [warp][stage][pass][16 bytes][lane]
    __shared__ float bufs[MODE == kAny ? kWarps : 1][256];
    constexpr int kPieces = sizeof(T) / 2, kStages = kFwdRing<T>;
    constexpr uint32_t kStage = kPasses * 256 * sizeof(T);
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
    char *const mine = ring + warp * (kStages * kStage) + lane * 16;
    const uint32_t mine_s = (uint32_t)__cvta_generic_to_shared(mine);
    auto fetch = [&](int b) {
        if (b < b1) {
            const int kind = kind_of(b), h0 = first_of(b, kind), n = in ? kind ? a.n_kv : a.n_q : 0;
            const Heads<const T> &x = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
            const T *at = x.at(t, h0) + f;
            const uint32_t to = mine_s + (b - b0) % kStages * kStage;
#pragma unroll
            for (int p = 0; p < kPasses; ++p, at += hp * x.head)
#pragma unroll
                for (int c = 0; c < kPieces; ++c)
                    copy16(to + (p * kPieces + c) * 512, h0 + p * hp < n ? at + 4 * c : x.p, h0 + p * hp < n);
        }
        copies_group();
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch(b0 + i);
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
    uint64_t tc[4], ts[4];  // factors
    int have = -1;          // of this kind
    for (int b = b0; b < b1; ++b) {
        const int kind = kind_of(b), h0 = first_of(b, kind), n = kind ? a.n_kv : a.n_q;
        fetch(b + kStages - 1);
        copies_wait<kStages - 1>();
        Raw<T> r[kPasses];
#pragma unroll
        for (int p = 0; p < kPasses; ++p) taken(r[p], mine + (b - b0) % kStages * kStage + p * kPieces * 512);
        if (APPEND && kind == 2) {
#pragma unroll
            for (int p = 0; p < kPasses; ++p)
                if (in && vc && h0 + p * hp < n) r[p].store(vc + (h0 + p * hp) * a.head + f);
        } else {
            const float *gain = kind ? a.gain_k : a.gain_q;
            Turn tn;
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
            if (kind != have) pack8(tc, tn.c), pack8(ts, tn.s);
            have = kind;
            float scale[kPasses];
#pragma unroll
            for (int p = 0; p < kPasses; ++p) scale[p] = 1.f;
            if (a.norm) {
#pragma unroll
                for (int p = 0; p < kPasses; ++p) {
                    uint64_t x[4], s = 0;
                    r[p].get(x);
#pragma unroll
                    for (int i = 0; i < 4; ++i) s = fma2(x[i], x[i], s);
                    scale[p] = sum2(s);
                }
                head_sums<LP>(scale, a.lp, lane);
#pragma unroll
                for (int p = 0; p < kPasses; ++p) scale[p] = rsqrtf(fmaf(scale[p], a.inv_d, a.eps));
            }
            if (!known)
#pragma unroll
                for (int p = 0; p < kPasses; ++p) r[p].zero(), scale[p] = 0.f;
            T *out = kind == 0 ? a.q_out.at(t, h0) + f : APPEND ? kc + h0 * a.head + f : a.k_out.at(t, h0) + f;
            const int64_t step = hp * (kind == 0 ? a.q_out.head : APPEND ? a.head : a.k_out.head);
            const int real = in && (!APPEND || kind == 0 || kc) ? n : 0;
#pragma unroll
            for (int p = 0; p < kPasses; ++p, out += step) {
                uint64_t x[4], y[4];
                float z[8];
                r[p].get(x);
                others<MODE>(y, r[p], f, a.rot, a.interleaved, bufs[MODE == kAny ? warp : 0], lane);
                const uint64_t s2 = pack2(scale[p], scale[p]);
#pragma unroll
                for (int i = 0; i < 4; ++i) unpack2(mul2(fma2(y[i], ts[i], mul2(x[i], tc[i])), s2), z[2 * i], z[2 * i + 1]);
                Raw<T> o;
                o.set(z);
                if (h0 + p * hp < real) o.store(out);
            }
        }
    }
}

// Persistent over the batches of the queries, then of the keys, so that a lane adds up its
// features' gain gradients in registers, the block in shared memory: one partial per block.
// Two batches per warp are on their way to shared memory while one is worked on, 128 KB per
// SM: in registers there is no room for more than the one.  16384 tokens of 16 + 16 heads of
// 128 features 78 us, 5.1 TB/s, with loads to registers 85 (and 100 with a butterfly per sum):
// reading and the issue of about 600 instructions a batch, four warps per scheduler.
constexpr int kRing = 3;
template <typename T> constexpr int kBwdBlocks = sizeof(T) == 2 ? 2 : 1;  // of an SM
template <typename T> constexpr uint32_t kRingBytes = kWarps * kRing * 2 * kPasses * 256 * sizeof(T);
template <int MODE, int LP, typename T>
__global__ void __launch_bounds__(32 * kWarps, kBwdBlocks<T>) bwd_kernel(const __grid_constant__ Args<T> a)
{
    extern __shared__ __align__(16) char ring[];  // [warp][stage][dy, x][pass][16 bytes][lane]
    __shared__ float bufs[kWarps][256];
    constexpr int kPieces = sizeof(T) / 2;  // of 16 bytes of a lane's features
    constexpr uint32_t kStage = 2 * kPasses * 256 * sizeof(T);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int lp = LP ? LP : a.lp, hp = 32 / lp, f = lane % lp * 8, own = lane / lp;
    const bool in = f < a.d;
    char *const mine = ring + warp * (kRing * kStage) + lane * 16;
    const uint32_t mine_s = (uint32_t)__cvta_generic_to_shared(mine);
    for (int kind = 0; kind < 2; ++kind) {
        const Heads<const T> &xs = kind ? a.k : a.q, &ds = kind ? a.dk : a.dq;
        const Heads<T> &out = kind ? a.k_out : a.q_out;
        const float *gain = kind ? a.gain_k : a.gain_q;
        const int n = kind ? a.n_kv : a.n_q, per = kind ? a.batches_kv : a.batches_q;
        float ones[8];
        uint64_t g[4], sum[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) ones[i] = 1.f;
        if (gain && in) load8(ones, gain + f);
        pack8(g, ones);
        // unit = (token, batch); a stride of the grid's warps is step_t tokens and step_b batches
        const int64_t u0 = (int64_t)blockIdx.x * kWarps + warp;
        const int stride = gridDim.x * kWarps, step_t = stride / per, step_b = stride - step_t * per;
        struct At {
            int64_t t;
            int b;
        };
        auto next = [&](At &x) {
            x.t += step_t, x.b += step_b;
            if (x.b >= per) x.b -= per, ++x.t;
        };
        const int real = in ? n : 0;
        auto fetch = [&](const At &x, int stage) {
            if (x.t < a.tokens) {
                const int h0 = x.b * kPasses * hp + own;
                const T *d_at = ds.at(x.t, h0) + f, *x_at = xs.at(x.t, h0) + f;
                const uint32_t to = mine_s + stage * kStage;
#pragma unroll
                for (int p = 0; p < kPasses; ++p, d_at += hp * ds.head, x_at += hp * xs.head) {
                    const bool r = h0 + p * hp < real;
#pragma unroll
                    for (int c = 0; c < kPieces; ++c) {
                        copy16(to + (p * kPieces + c) * 512, r ? d_at + 4 * c : ds.p, r);
                        if (a.norm) copy16(to + ((kPasses + p) * kPieces + c) * 512, r ? x_at + 4 * c : xs.p, r);
                    }
                }
            }
            copies_group();
        };
        At at{u0 / per, 0};
        at.b = (int)(u0 - at.t * per);
        At ahead = at;
        int stage = 0;
#pragma unroll
        for (int i = 0; i < kRing - 1; ++i) fetch(ahead, i), next(ahead);
        int pos = at.t < a.tokens ? a.pos[at.t] : 0;
        while (at.t < a.tokens) {
            fetch(ahead, stage ? stage - 1 : kRing - 1);
            next(ahead);
            const int64_t t = at.t;
            const int h0 = at.b * kPasses * hp + own;
            const bool known = pos >= 0 && pos < a.positions;
            if (!known && lane == 0) raise_status(a.status, kStatusBadIndex);
            Turn tn;
            load_turn<MODE, -1>(tn, a.table + (int64_t)(known ? pos : 0) * a.rot, known && in ? f : a.rot, a.rot, a.interleaved);
            next(at);
            if (at.t < a.tokens) pos = a.pos[at.t];
            copies_wait<kRing - 1>();
            Raw<T> rx[kPasses], rd[kPasses];
#pragma unroll
            for (int p = 0; p < kPasses; ++p) {
                taken(rd[p], mine + stage * kStage + p * kPieces * 512);
                if (a.norm) taken(rx[p], mine + stage * kStage + (kPasses + p) * kPieces * 512);
            }
            stage = stage == kRing - 1 ? 0 : stage + 1;
            uint64_t tc[4], ts[4];
            pack8(tc, tn.c), pack8(ts, tn.s);
            if (!known)  // the forward's outputs are 0 whatever x holds
#pragma unroll
                for (int p = 0; p < kPasses; ++p) rd[p].zero(), rx[p].zero();
            auto turned = [&](uint64_t (&w)[4], int p) {
                uint64_t y[4];
                rd[p].get(w);
                others<MODE>(y, rd[p], f, a.rot, a.interleaved, bufs[warp], lane);
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = fma2(y[i], ts[i], mul2(w[i], tc[i]));
            };
            uint64_t w[kPasses][4];
            float v[2 * kPasses];  // sums of x², then of g w x
#pragma unroll
            for (int p = 0; p < kPasses; ++p) {
                turned(w[p], p);
                if (!a.norm) continue;
                uint64_t x[4], xx = 0, wx = 0;
                rx[p].get(x);
#pragma unroll
                for (int i = 0; i < 4; ++i) xx = fma2(x[i], x[i], xx), wx = fma2(mul2(w[p][i], g[i]), x[i], wx);
                v[p] = sum2(xx), v[kPasses + p] = sum2(wx);
            }
            if (a.norm) head_sums<LP>(v, a.lp, lane);
            T *o_at = out.at(t, h0) + f;
#pragma unroll
            for (int p = 0; p < kPasses; ++p, o_at += hp * out.head) {
                if (a.norm) {
                    uint64_t x[4];
                    rx[p].get(x);
                    const float scale = rsqrtf(fmaf(v[p], a.inv_d, a.eps)), c = -(v[kPasses + p] * scale * a.inv_d * scale) * scale;
                    const uint64_t s2 = pack2(scale, scale), c2 = pack2(c, c);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        sum[i] = fma2(mul2(w[p][i], x[i]), s2, sum[i]);  // 0 in lanes without a head
                        w[p][i] = fma2(x[i], c2, mul2(mul2(w[p][i], g[i]), s2));
                    }
                }
                float z[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) unpack2(w[p][i], z[2 * i], z[2 * i + 1]);
                Raw<T> o;
                o.set(z);
                if (h0 + p * hp < real) o.store(o_at);
            }
        }
        copies_wait<0>();
        if (!a.part) continue;
        // over the heads side by side in the warp, then over the warps, in order
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack2(sum[i], bufs[warp][lane * 8 + 2 * i], bufs[warp][lane * 8 + 2 * i + 1]);
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
