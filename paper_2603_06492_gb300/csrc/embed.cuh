// Rows of a table by token, and the table's gradient.
//
//   y[t] = scale table[id[t]]
//   dtable[v] = scale * sum over the tokens t with id[t] = v of dy[t], t ascending
//
// The gradient writes every row of the table, zeros included, which is most of its traffic
// when the table is large.  Tokens are brought into the order of their numbers first; what
// the order of atomics decides (places of the lists of tokens, and orders within them) is
// undone before anything is added up, so that sums do not depend on it.
#pragma once

#include "norm.cuh"

namespace noble {
namespace embed {

using norm::Vec;

template <typename T>
struct FwdArgs {
    const int32_t *ids;
    const T *table;
    T *y;
    int64_t tokens;
    int vocab, d;
    float scale;
    uint32_t *status;
};

// One warp per token and piece of 32 NV vectors of its row.
template <typename T, int NV>
__global__ void __launch_bounds__(256) fwd_kernel(const FwdArgs<T> a)
{
    constexpr int V = Vec<T>::n;
    const int lane = threadIdx.x % 32, vecs = a.d / V;
    const int64_t t = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
    if (t >= a.tokens) return;
    const int id = a.ids[t];
    const bool bad = id >= a.vocab;
    if (bad && lane == 0 && blockIdx.y == 0) raise_status(a.status, kStatusBadIndex);
    const bool there = id >= 0 && !bad;
    const uint4 *src = reinterpret_cast<const uint4 *>(a.table + (there ? (int64_t)id * a.d : 0));
    uint4 *dst = reinterpret_cast<uint4 *>(a.y + t * a.d);
    for (int at = blockIdx.y * 32 * NV + lane; at < vecs; at += gridDim.y * 32 * NV) {
        uint4 q[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            q[i] = make_uint4(0, 0, 0, 0);
            if (there && at + 32 * i < vecs) q[i] = src[at + 32 * i];
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (at + 32 * i < vecs) {
                if (a.scale != 1.f) {
                    float f[V];
                    Vec<T>::unpack(q[i], f);
#pragma unroll
                    for (int j = 0; j < V; ++j) f[j] *= there ? a.scale : 0.f;
                    q[i] = Vec<T>::pack(f);
                }
                dst[at + 32 * i] = q[i];
            }
    }
}

// ---------------------------------------------------------------- gradient
constexpr int kFewTokens = 2048;  // at most so many: one launch
constexpr int kFewRows = 64;      // rows of the table of a block then
constexpr int kShort = 32;        // a list of so many tokens is one warp's
constexpr int kPiece = 64;        // tokens of a piece of a longer list
constexpr int kWindow = 1 << 18;  // tokens that a block's bit map covers at a time

template <typename T>
struct BwdArgs {
    const int32_t *ids;
    const T *dy;
    float *dtable;
    int64_t tokens;
    int vocab, d;
    float scale;
    uint32_t *status;
    // many tokens: tokens of each row, where its list begins, each token's place in it
    uint32_t *count, *begin, *rank, *list;
    uint32_t *head;      // [0] tokens listed, [1] long lists, [2] pieces
    uint32_t *long_row;  // rows with long lists
    uint32_t *long_at;   // their first pieces
    uint2 *piece;        // row, which piece of its list
    float *part;         // [pieces][d]
};

// acc += the rows of dy that list names, first to last; the columns of vector `at`
template <typename T>
__device__ __forceinline__ void add_rows(const T *dy, int64_t d, const uint32_t *list, int n, int at, float (&acc)[Vec<T>::n])
{
    constexpr int V = Vec<T>::n, kAhead = 8;
    int k = 0;
    for (; k + kAhead <= n; k += kAhead) {
        uint4 q[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) q[i] = reinterpret_cast<const uint4 *>(dy + (int64_t)list[k + i] * d)[at];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            float f[V];
            Vec<T>::unpack(q[i], f);
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] += f[j];
        }
    }
    for (; k < n; ++k) {
        float f[V];
        Vec<T>::unpack(reinterpret_cast<const uint4 *>(dy + (int64_t)list[k] * d)[at], f);
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += f[j];
    }
}
template <int N>
__device__ __forceinline__ void store_scaled(float *p, const float (&f)[N], float scale)
{
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
        __stcs(reinterpret_cast<float4 *>(p) + i,
               make_float4(f[4 * i] * scale, f[4 * i + 1] * scale, f[4 * i + 2] * scale, f[4 * i + 3] * scale));
}

// Few tokens: a block has kFewRows rows of the table and 32 vectors of their columns, finds
// the tokens of its rows in ascending order and adds them up, a row to a warp.
template <typename T>
__global__ void __launch_bounds__(256) few_kernel(const BwdArgs<T> a)
{
    constexpr int V = Vec<T>::n;
    __shared__ uint32_t found[kFewTokens];  // row of the block << 16 | token
    __shared__ uint32_t mine[8][kFewTokens / 4];
    __shared__ int counts[8];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int first = blockIdx.x * kFewRows, rows = min(kFewRows, a.vocab - first), n = (int)a.tokens;
    const int at = blockIdx.y * 32 + lane;
    const bool in = at < a.d / V;
    int total = 0;
    for (int t0 = 0; t0 < n; t0 += 256) {
        const int t = t0 + threadIdx.x;
        const int id = t < n ? a.ids[t] : -1;
        if (id >= a.vocab && blockIdx.x == 0 && blockIdx.y == 0) raise_status(a.status, kStatusBadIndex);
        const bool hit = id >= first && id < first + rows;
        const uint32_t mask = __ballot_sync(0xffffffffu, hit);
        if (lane == 0) counts[warp] = __popc(mask);
        __syncthreads();
        int before = total;
        for (int w = 0; w < 8; ++w) {
            if (w < warp) before += counts[w];
            total += counts[w];
        }
        if (hit) found[before + __popc(mask & ((1u << lane) - 1))] = (uint32_t)(id - first) << 16 | (uint32_t)t;
        __syncthreads();
    }
    for (int r = warp; r < rows; r += 8) {
        float acc[V];
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.f;
        // this row's tokens, a quarter of the longest list at a time
        int k = 0;
        while (k < total) {
            int m = 0;
            for (; k < total && m + 32 <= kFewTokens / 4; k += 32) {
                const uint32_t e = k + lane < total ? found[k + lane] : ~0u;
                const bool hit = e >> 16 == (uint32_t)r;
                const uint32_t mask = __ballot_sync(0xffffffffu, hit);
                if (hit) mine[warp][m + __popc(mask & ((1u << lane) - 1))] = e & 0xffffu;
                m += __popc(mask);
            }
            __syncwarp();
            if (in) add_rows(a.dy, a.d, mine[warp], m, at, acc);
            __syncwarp();
        }
        if (in) store_scaled(a.dtable + (int64_t)(first + r) * a.d + at * V, acc, a.scale);
    }
}

// ---- many tokens
// tokens of each row, and each token's place among them (which atomics decide)
template <typename T>
__global__ void __launch_bounds__(256) count_kernel(const BwdArgs<T> a)
{
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    int id = t < a.tokens ? a.ids[t] : -1;
    if (id >= a.vocab) {
        raise_status(a.status, kStatusBadIndex);
        id = -1;
    }
    // one atomic for the lanes that share a row
    const uint32_t same = __match_any_sync(0xffffffffu, id);
    const int lead = __ffs(same) - 1, lane = threadIdx.x % 32;
    uint32_t base = 0;
    if (id >= 0 && lane == lead) base = atomicAdd(a.count + id, (uint32_t)__popc(same));
    base = __shfl_sync(0xffffffffu, base, lead);
    if (t < a.tokens) a.rank[t] = id < 0 ? ~0u : base + __popc(same & ((1u << lane) - 1));
}

// where each row's list begins; long lists and their pieces
template <typename T>
__global__ void __launch_bounds__(256) lists_kernel(const BwdArgs<T> a)
{
    const int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int lane = threadIdx.x % 32;
    const uint32_t n = v < a.vocab ? a.count[v] : 0;
    uint32_t upto = n;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += u;
    }
    uint32_t base = 0;
    if (lane == 31 && upto) base = atomicAdd(a.head, upto);
    base = __shfl_sync(0xffffffffu, base, 31);
    if (v < a.vocab) a.begin[v] = base + upto - n;
    if (n > kShort) {
        const uint32_t l = atomicAdd(a.head + 1, 1u), pieces = (n + kPiece - 1) / kPiece, p = atomicAdd(a.head + 2, pieces);
        a.long_row[l] = (uint32_t)v;
        a.long_at[l] = p;
        for (uint32_t k = 0; k < pieces; ++k) a.piece[p + k] = make_uint2((uint32_t)v, k);
    }
}

template <typename T>
__global__ void __launch_bounds__(256) place_kernel(const BwdArgs<T> a)
{
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= a.tokens) return;
    const uint32_t r = a.rank[t];
    if (r != ~0u) a.list[a.begin[a.ids[t]] + r] = (uint32_t)t;
}

// Long lists in ascending order: a bit for each token, read off again word by word.  The
// tokens of a window are listed before those of the next; `rank`, which nothing needs any
// more, takes the ordered list.
template <typename T>
__global__ void __launch_bounds__(256) order_kernel(const BwdArgs<T> a)
{
    extern __shared__ uint32_t bits[];
    __shared__ uint32_t sums[8];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (uint32_t l = blockIdx.x; l < a.head[1]; l += gridDim.x) {
        const uint32_t row = a.long_row[l], n = a.count[row], begin = a.begin[row];
        uint32_t done = begin;
        for (int64_t w0 = 0; w0 < a.tokens; w0 += kWindow) {
            const int words = (int)((min((int64_t)kWindow, a.tokens - w0) + 31) / 32);
            for (int i = threadIdx.x; i < words; i += 256) bits[i] = 0;
            __syncthreads();
            for (uint32_t k = threadIdx.x; k < n; k += 256) {
                const int64_t t = (int64_t)a.list[begin + k] - w0;
                if (t >= 0 && t < kWindow) atomicOr(bits + t / 32, 1u << (t % 32));
            }
            __syncthreads();
            for (int i0 = 0; i0 < words; i0 += 256) {
                const int i = i0 + threadIdx.x;
                uint32_t b = i < words ? bits[i] : 0;
                const uint32_t c = __popc(b);
                uint32_t upto = c;
#pragma unroll
                for (int o = 1; o < 32; o *= 2) {
                    const uint32_t u = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += u;
                }
                if (lane == 31) sums[warp] = upto;
                __syncthreads();
                uint32_t at = done + upto - c;
                for (int w = 0; w < 8; ++w) {
                    if (w < warp) at += sums[w];
                    done += sums[w];
                }
                for (; b; b &= b - 1) a.rank[at++] = (uint32_t)(w0 + 32 * i + __ffs(b) - 1);
                __syncthreads();
            }
        }
    }
}

// A warp per row with a short list, or none, and per piece of a long one: the rows come
// first, then the pieces.  blockIdx.y: columns, 32 vectors at a time.
template <typename T>
__global__ void __launch_bounds__(256) sum_kernel(const BwdArgs<T> a)
{
    constexpr int V = Vec<T>::n;
    __shared__ uint32_t order[8][kPiece];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, vecs = a.d / V;
    const int64_t work = (int64_t)a.vocab + a.head[2];
    for (int64_t w = (int64_t)blockIdx.x * 8 + warp; w < work; w += (int64_t)gridDim.x * 8) {
        int n;
        float *out;
        __syncwarp();
        if (w < a.vocab) {
            n = (int)a.count[w];
            if (n > kShort) continue;
            out = a.dtable + w * a.d;
            const uint32_t t = lane < n ? a.list[a.begin[w] + lane] : ~0u;
            // a token's place: how many of the list come before it
            int place = 0;
            for (int k = 0; k < n; ++k) place += __shfl_sync(0xffffffffu, t, k) < t;
            if (lane < n) order[warp][place] = t;
        } else {
            const uint2 p = a.piece[w - a.vocab];
            const uint32_t begin = a.begin[p.x] + p.y * kPiece;
            n = (int)min((uint32_t)kPiece, a.count[p.x] - p.y * kPiece);
            out = a.part + (w - a.vocab) * a.d;
            for (int k = lane; k < n; k += 32) order[warp][k] = a.rank[begin + k];
        }
        __syncwarp();
        for (int at = blockIdx.y * 32 + lane; at < vecs; at += gridDim.y * 32) {
            float acc[V];
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] = 0.f;
            add_rows(a.dy, a.d, order[warp], n, at, acc);
            store_scaled(out + at * V, acc, w < a.vocab ? a.scale : 1.f);
        }
    }
}

// the pieces of each long list, first to last
template <typename T>
__global__ void __launch_bounds__(256) join_kernel(const BwdArgs<T> a)
{
    const int quads = a.d / 4;
    for (uint32_t l = blockIdx.x; l < a.head[1]; l += gridDim.x) {
        const uint32_t row = a.long_row[l], pieces = (a.count[row] + kPiece - 1) / kPiece;
        const float *part = a.part + (int64_t)a.long_at[l] * a.d;
        for (int at = blockIdx.y * 256 + threadIdx.x; at < quads; at += gridDim.y * 256) {
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
            for (uint32_t k = 0; k < pieces; ++k) {
                const float4 q = reinterpret_cast<const float4 *>(part + (int64_t)k * a.d)[at];
                acc[0] += q.x, acc[1] += q.y, acc[2] += q.z, acc[3] += q.w;
            }
            store_scaled(a.dtable + (int64_t)row * a.d + 4 * at, acc, a.scale);
        }
    }
}

}  // namespace embed
}  // namespace noble
