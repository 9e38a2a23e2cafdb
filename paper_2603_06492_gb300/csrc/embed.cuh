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
// 32 bytes a lane in one store where they are aligned: two of 16 write every sector twice.
template <int N>
__device__ __forceinline__ void store_scaled(float *p, const float (&f)[N], float scale, bool wide)
{
    if constexpr (N == 8) {
        if (wide) {
            asm volatile("st.global.cs.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(f[0] * scale), "f"(f[1] * scale),
                         "f"(f[2] * scale), "f"(f[3] * scale), "f"(f[4] * scale), "f"(f[5] * scale), "f"(f[6] * scale),
                         "f"(f[7] * scale)
                         : "memory");
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
        __stcs(reinterpret_cast<float4 *>(p) + i,
               make_float4(f[4 * i] * scale, f[4 * i + 1] * scale, f[4 * i + 2] * scale, f[4 * i + 3] * scale));
}

constexpr int kFewTokens = 1024;  // at most so many: one launch
constexpr int kFewRows = 64;      // rows of the table of a block then
constexpr int kFewAlone = 16;     // tokens of a row that one warp adds up
constexpr int kShort = 8;         // a list of so many tokens is one warp's
constexpr int kPiece = 64;        // tokens of a piece of a longer list
constexpr int kCompared = 256;    // tokens of a list that is ordered by comparing
constexpr int kWindow = 1 << 18;  // tokens that a block's bit map covers at a time, for longer ones

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
    uint32_t *head;      // [0] tokens listed, [1] long lists, [2] their pieces, [3] of several, [4] lists of several
    uint32_t *long_row;  // rows with long lists
    uint2 *piece;        // row, which piece of its list
    uint32_t *piece_part;  // where the piece's sum goes in `part`; ~0: a list of one piece, to the table
    uint2 *joined;       // lists of several pieces: row, first of their sums
    float *part;         // [pieces of lists of several][d]
    int rows_per_warp, piece_blocks;  // of sum_kernel
    int wide, part_wide;  // dtable, part are aligned to 32 bytes: the interface asks for 16
};

// out = scale * (the sum of the n rows of dy that list names, first to last), the columns of vectors at,
// at + 32, ..., C of them: B tokens' loads are on their way at once.  wide: `out` is aligned to 32 bytes.
template <int C, int B, typename T>
__device__ __forceinline__ void sum_vectors(const BwdArgs<T> &a, const uint32_t *list, int n, int at, float *out, float scale, bool wide)
{
    constexpr int V = Vec<T>::n;
    const int vecs = a.d / V;
    float acc[C][V];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[c][j] = 0.f;
    for (int k = 0; k < n; k += B) {
        uint4 q[B][C];
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const uint4 *row = reinterpret_cast<const uint4 *>(a.dy + (k + i < n ? (int64_t)list[k + i] * a.d : 0));
#pragma unroll
            for (int c = 0; c < C; ++c) q[i][c] = k + i < n && at + 32 * c < vecs ? row[at + 32 * c] : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < B; ++i)
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float f[V];
                Vec<T>::unpack(q[i][c], f);
#pragma unroll
                for (int j = 0; j < V; ++j) acc[c][j] += f[j];
            }
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
        if (at + 32 * c < vecs) store_scaled(out + (at + 32 * c) * V, acc[c], scale, wide);
}
// ... of all vectors of a row of the table from `at` on that are `step` apart, but for the steps within a
// warp; n <= kShort.
template <typename T>
__device__ __forceinline__ void sum_row(const BwdArgs<T> &a, const uint32_t *list, int n, int at, int step, float *out, float scale)
{
    const int vecs = a.d / Vec<T>::n;
    if (step != 32) {
        for (; at < vecs; at += step) sum_vectors<1, 8>(a, list, n, at, out, scale, a.wide);
    } else if (n <= 2) {
        for (; at < vecs; at += 4 * 32) sum_vectors<4, 2>(a, list, n, at, out, scale, a.wide);
    } else {
        for (; at < vecs; at += 2 * 32) sum_vectors<2, 4>(a, list, n, at, out, scale, a.wide);
    }
}

// Few tokens: a block has kFewRows rows of the table and 32 vectors of their columns, finds
// the tokens of its rows in ascending order and adds them up, a row to a warp.
template <typename T>
__global__ void __launch_bounds__(256) few_kernel(const BwdArgs<T> a)
{
    constexpr int V = Vec<T>::n;
    __shared__ uint32_t found[kFewTokens];  // row of the block << 16 | token
    __shared__ uint32_t mine[8][kFewTokens / 8];
    __shared__ int counts[8], many[kFewRows];
    __shared__ float sums[8][V][32];
    if (threadIdx.x < kFewRows) many[threadIdx.x] = 0;
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
        if (hit) {
            found[before + __popc(mask & ((1u << lane) - 1))] = (uint32_t)(id - first) << 16 | (uint32_t)t;
            atomicAdd(many + id - first, 1);
        }
        __syncthreads();
    }
    const bool crowded = __syncthreads_or(threadIdx.x < kFewRows && many[threadIdx.x] > kFewAlone);
    // a row's tokens among found[from .. to), over the warp's part of `mine` again and again
    auto add = [&](int r, int from, int to, float (&acc)[V]) {
        for (int k = from; k < to;) {
            int m = 0;
            for (; k < to && m + 32 <= kFewTokens / 8; k += 32) {
                const uint32_t e = k + lane < to ? found[k + lane] : ~0u;
                const bool hit = e >> 16 == (uint32_t)r;
                const uint32_t mask = __ballot_sync(0xffffffffu, hit);
                if (hit) mine[warp][m + __popc(mask & ((1u << lane) - 1))] = e & 0xffffu;
                m += __popc(mask);
            }
            __syncwarp();
            for (int i0 = 0; in && i0 < m; i0 += 8) {
                uint4 q[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    q[i] = i0 + i < m ? reinterpret_cast<const uint4 *>(a.dy + (int64_t)mine[warp][i0 + i] * a.d)[at] : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float f[V];
                    Vec<T>::unpack(q[i], f);
#pragma unroll
                    for (int j = 0; j < V; ++j) acc[j] += f[j];
                }
            }
            __syncwarp();
        }
    };
    for (int r = warp; r < rows; r += 8) {
        if (many[r] > kFewAlone) continue;
        float acc[V] = {};
        if (many[r]) add(r, 0, total, acc);
        if (in) store_scaled(a.dtable + (int64_t)(first + r) * a.d + at * V, acc, a.scale, a.wide);
    }
    // rows of more tokens: an eighth of what was found to a warp, then the eighths in order
    for (int r = 0; crowded && r < rows; ++r) {
        if (many[r] <= kFewAlone) continue;
        const int per = (total + 7) / 8;
        float acc[V] = {};
        add(r, warp * per, min(total, (warp + 1) * per), acc);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < V; ++j) sums[warp][j][lane] = acc[j];
        __syncthreads();
        if (warp != 0 || !in) continue;
#pragma unroll
        for (int j = 0; j < V; ++j)
            for (int w = 1; w < 8; ++w) acc[j] += sums[w][j][lane];
        store_scaled(a.dtable + (int64_t)(first + r) * a.d + at * V, acc, a.scale, a.wide);
    }
}

// ---- many tokens
// Three steps make a list of the tokens of each row, each step over everything that the one before
// it wrote; `thread` of `threads` in whole warps.

// tokens of each row, and each token's place among them (which atomics decide)
template <typename T>
__device__ __forceinline__ void count_tokens(const BwdArgs<T> &a, int64_t thread, int64_t threads)
{
    const int lane = threadIdx.x % 32;
    for (int64_t t = thread; t - lane < a.tokens; t += threads) {
        int id = t < a.tokens ? a.ids[t] : -1;
        if (id >= a.vocab) {
            raise_status(a.status, kStatusBadIndex);
            id = -1;
        }
        // one atomic for the lanes that share a row
        const uint32_t same = __match_any_sync(0xffffffffu, id);
        const int lead = __ffs(same) - 1;
        uint32_t base = 0;
        if (id >= 0 && lane == lead) base = atomicAdd(a.count + id, (uint32_t)__popc(same));
        base = __shfl_sync(0xffffffffu, base, lead);
        if (t < a.tokens) a.rank[t] = id < 0 ? ~0u : base + __popc(same & ((1u << lane) - 1));
    }
}

// where each row's list begins, eight rows to a thread; long lists and their pieces
template <typename T>
__device__ __forceinline__ void begin_lists(const BwdArgs<T> &a, int64_t thread, int64_t threads)
{
    const int lane = threadIdx.x % 32;
    for (int64_t v = 8 * thread; v - 8 * lane < a.vocab; v += 8 * threads) {
        uint32_t n[8], mine = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint4 q = make_uint4(0, 0, 0, 0);
            if (v + 4 * h < a.vocab) q = __ldcg(reinterpret_cast<const uint4 *>(a.count + v) + h);
            n[4 * h] = q.x, n[4 * h + 1] = q.y, n[4 * h + 2] = q.z, n[4 * h + 3] = q.w;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (v + i >= a.vocab) n[i] = 0;  // behind the last row
            mine += n[i];
        }
        // room for this warp's tokens, lists, pieces: sums over the lanes, one atomic for each kind
        uint32_t kinds[5] = {mine, 0, 0, 0, 0}, base[5];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (n[i] <= kShort) continue;
            const uint32_t pieces = (n[i] + kPiece - 1) / kPiece;
            kinds[1] += 1, kinds[2] += pieces;
            if (pieces > 1) kinds[3] += pieces, kinds[4] += 1;
        }
        const bool some_long = __any_sync(0xffffffffu, kinds[1]);
        const int live = some_long ? 5 : 1;
        uint32_t total = 0;  // in lane k, of kind k
#pragma unroll
        for (int k = 0; k < 5; ++k) {
            if (k >= live) break;
            uint32_t upto = kinds[k];
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const uint32_t u = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += u;
            }
            const uint32_t all = __shfl_sync(0xffffffffu, upto, 31);
            if (lane == k) total = all;
            base[k] = upto - kinds[k];
        }
        uint32_t room = 0;
        if (total) room = atomicAdd(a.head + lane, total);
#pragma unroll
        for (int k = 0; k < 5; ++k)
            if (k < live) base[k] += __shfl_sync(0xffffffffu, room, k);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t c = n[i], row = (uint32_t)(v + i);
            if (!c) continue;
            a.begin[v + i] = base[0];
            base[0] += c;
            if (c <= kShort) continue;
            const uint32_t pieces = (c + kPiece - 1) / kPiece;
            a.long_row[base[1]++] = row;
            if (pieces > 1) a.joined[base[4]++] = make_uint2(row, base[3]);
            for (uint32_t k = 0; k < min(pieces, 4u); ++k) {
                a.piece[base[2] + k] = make_uint2(row, k);
                a.piece_part[base[2] + k] = pieces > 1 ? base[3] + k : ~0u;
            }
            base[2] += pieces;
            if (pieces > 1) base[3] += pieces;
        }
        // pieces after a list's fourth by the whole warp
#pragma unroll
        for (int i = 0; some_long && i < 8; ++i) {
            for (uint32_t more = __ballot_sync(0xffffffffu, n[i] > 4 * kPiece); more; more &= more - 1) {
                const int from = __ffs(more) - 1;
                const uint32_t pieces = (__shfl_sync(0xffffffffu, n[i], from) + kPiece - 1) / kPiece;
                // behind this list's, the lane has put those of its later rows
                uint32_t after2 = 0, after3 = 0;
#pragma unroll
                for (int j = i + 1; j < 8; ++j) {
                    const uint32_t p = n[j] > kShort ? (n[j] + kPiece - 1) / kPiece : 0;
                    after2 += p, after3 += p > 1 ? p : 0;
                }
                const uint32_t at2 = __shfl_sync(0xffffffffu, base[2] - after2, from) - pieces;
                const uint32_t at3 = __shfl_sync(0xffffffffu, base[3] - after3, from) - pieces;
                const uint32_t row = (uint32_t)__shfl_sync(0xffffffffu, (int)v, from) + i;
                for (uint32_t k = 4 + lane; k < pieces; k += 32) {
                    a.piece[at2 + k] = make_uint2(row, k);
                    a.piece_part[at2 + k] = at3 + k;
                }
            }
        }
    }
}

template <typename T>
__device__ __forceinline__ void place_tokens(const BwdArgs<T> &a, int64_t thread, int64_t threads)
{
    for (int64_t t = thread; t < a.tokens; t += threads) {
        const uint32_t r = __ldcg(a.rank + t);
        if (r != ~0u) a.list[__ldcg(a.begin + a.ids[t]) + r] = (uint32_t)t;
    }
}

// Long lists in ascending order, a list to a block at a time; `rank`, which nothing needs any more,
// takes them.  Up to kCompared tokens each token's place is the number of smaller ones; beyond,
// a bit is set for each token and the bits are read off again word by word, the tokens of a window
// before those of the next.  Each window goes over the whole list: one row with all of 2^20 tokens takes 2.2 ms, with
// 2^24 225; 2^24 tokens spread over 100 rows 9 ms.
template <typename T>
__global__ void __launch_bounds__(256) order_kernel(const BwdArgs<T> a)
{
    extern __shared__ uint32_t bits[];
    __shared__ uint32_t sums[8];
    __shared__ __align__(16) uint32_t some[kCompared];
    ptx::griddep_launch();
    ptx::griddep_wait();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const uint32_t lists = a.head[1];
    for (uint32_t l = blockIdx.x; l < lists; l += gridDim.x) {
        const uint32_t row = a.long_row[l], n = a.count[row], begin = a.begin[row];
        if (n <= kCompared) {
            const uint32_t t = threadIdx.x < n ? a.list[begin + threadIdx.x] : ~0u;
            __syncthreads();
            some[threadIdx.x] = t;
            __syncthreads();
            uint32_t place = 0;
            for (uint32_t k = 0; k < n; k += 4) {  // what pads the last four is not smaller
                const uint4 q = *reinterpret_cast<const uint4 *>(some + k);
                place += (q.x < t) + (q.y < t) + (q.z < t) + (q.w < t);
            }
            if (threadIdx.x < n) a.rank[begin + place] = t;
            continue;
        }
        uint32_t done = begin;
        for (int64_t w0 = 0; w0 < a.tokens; w0 += kWindow) {
            const int words = (int)((min((int64_t)kWindow, a.tokens - w0) + 31) / 32);
            __syncthreads();
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

// The first three by one cluster of eight blocks, which wait for each other at the cluster's barrier.
constexpr int kIndexBlocks = 8, kIndexThreads = 1024;
constexpr int64_t kIndexTokens = 1 << 14, kIndexRows = 1 << 16;  // beyond, a launch each
template <typename T>
__global__ void __cluster_dims__(kIndexBlocks, 1, 1) __launch_bounds__(kIndexThreads) index_kernel(const BwdArgs<T> a)
{
    ptx::griddep_launch();
    ptx::griddep_wait();
    const int64_t thread = blockIdx.x * kIndexThreads + threadIdx.x, threads = kIndexBlocks * kIndexThreads;
    auto all = [] {
        __threadfence();
        __syncthreads();
        cluster::sync();
    };
    for (int64_t v = thread; 4 * v < a.vocab; v += threads) reinterpret_cast<uint4 *>(a.count)[v] = make_uint4(0, 0, 0, 0);
    if (thread < 8) a.head[thread] = 0;
    all();
    count_tokens(a, thread, threads);
    all();
    begin_lists(a, thread, threads);
    all();
    place_tokens(a, thread, threads);
}

template <typename T>
__global__ void __launch_bounds__(256) count_kernel(const BwdArgs<T> a)
{
    ptx::griddep_launch();
    ptx::griddep_wait();
    count_tokens(a, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}
template <typename T>
__global__ void __launch_bounds__(256) lists_kernel(const BwdArgs<T> a)
{
    ptx::griddep_launch();
    ptx::griddep_wait();
    begin_lists(a, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}
template <typename T>
__global__ void __launch_bounds__(256) place_kernel(const BwdArgs<T> a)
{
    ptx::griddep_launch();
    ptx::griddep_wait();
    place_tokens(a, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}
// A warp for rows_per_warp rows of the table with short lists, or none; the first blocks take the
// pieces of long lists.  blockIdx.y: columns, 32 vectors at a time.
template <typename T>
__global__ void __launch_bounds__(256) sum_kernel(const BwdArgs<T> a)
{
    constexpr int V = Vec<T>::n;
    __shared__ uint32_t order[8][kPiece];
    ptx::griddep_launch();
    ptx::griddep_wait();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, vecs = a.d / V;
    const int at0 = blockIdx.y * 32 + lane, step = gridDim.y * 32;
    if ((int)blockIdx.x < a.piece_blocks) {
        if (blockIdx.y) return;
        // 32 vectors of a piece to a warp
        const uint32_t slices = (vecs + 31) / 32;
        const uint64_t work = (uint64_t)a.head[2] * slices;
        for (uint64_t w = blockIdx.x * 8 + warp; w < work; w += (uint64_t)a.piece_blocks * 8) {
            const uint32_t piece = (uint32_t)(w / slices), part = a.piece_part[piece];
            const uint2 p = a.piece[piece];
            const uint32_t begin = a.begin[p.x] + p.y * kPiece;
            const int n = (int)min((uint32_t)kPiece, a.count[p.x] - p.y * kPiece), at = (int)(w - (uint64_t)piece * slices) * 32 + lane;
            __syncwarp();
            for (int k = lane; k < n; k += 32) order[warp][k] = a.rank[begin + k];
            __syncwarp();
            const bool whole = part == ~0u;
            float *out = whole ? a.dtable + (int64_t)p.x * a.d : a.part + (int64_t)part * a.d;
            if (at < vecs) sum_vectors<1, 8>(a, order[warp], n, at, out, whole ? a.scale : 1.f, whole ? a.wide : a.part_wide);
        }
        return;
    }
    // counts of this warp's rows, a lane each
    const int64_t first = ((int64_t)(blockIdx.x - a.piece_blocks) * 8 + warp) * a.rows_per_warp;
    const bool mine = lane < a.rows_per_warp && first + lane < a.vocab;
    const uint32_t count = mine ? a.count[first + lane] : ~0u;
    const uint32_t begin = mine && count && count <= kShort ? a.begin[first + lane] : 0;
    // rows without tokens, then the others: writing zeros waits for nothing
    for (uint32_t none = __ballot_sync(0xffffffffu, count == 0); none; none &= none - 1) {
        float *out = a.dtable + (first + __ffs(none) - 1) * a.d;
        const float zero[V] = {};
        for (int at = at0; at < vecs; at += step) store_scaled(out + at * V, zero, 1.f, a.wide);
    }
    for (uint32_t some = __ballot_sync(0xffffffffu, count && count <= kShort); some; some &= some - 1) {
        const int r = __ffs(some) - 1, n = (int)__shfl_sync(0xffffffffu, count, r);
        const uint32_t b = __shfl_sync(0xffffffffu, begin, r);
        const uint32_t t = lane < n ? a.list[b + lane] : ~0u;
        // a token's place: how many of the list come before it
        int place = 0;
        for (int k = 0; k < n; ++k) place += __shfl_sync(0xffffffffu, t, k) < t;
        __syncwarp();
        if (lane < n) order[warp][place] = t;
        __syncwarp();
        sum_row(a, order[warp], n, at0, step, a.dtable + (first + r) * a.d, a.scale);
    }
}

// The pieces of each list of several: 128 columns of a list to a block, an eighth of the pieces to a
// warp, in order; then the eighths in order.
template <typename T>
__global__ void __launch_bounds__(256) join_kernel(const BwdArgs<T> a)
{
    __shared__ float4 sm[8][32];
    ptx::griddep_wait();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, quads = a.d / 4;
    for (uint32_t l = blockIdx.x; l < a.head[4]; l += gridDim.x) {
        const uint32_t row = a.joined[l].x, pieces = (a.count[row] + kPiece - 1) / kPiece, per = (pieces + 7) / 8;
        const float *part = a.part + (int64_t)a.joined[l].y * a.d;
        for (int q0 = blockIdx.y * 32; q0 < quads; q0 += gridDim.y * 32) {
            const int at = q0 + lane;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            if (at < quads) {
                const uint32_t end = min(pieces, (warp + 1) * per);
#pragma unroll 8
                for (uint32_t k = warp * per; k < end; ++k) {
                    const float4 q = reinterpret_cast<const float4 *>(part + (int64_t)k * a.d)[at];
                    acc.x += q.x, acc.y += q.y, acc.z += q.z, acc.w += q.w;
                }
            }
            __syncthreads();
            sm[warp][lane] = acc;
            __syncthreads();
            if (warp == 0 && at < quads) {
                for (int w = 1; w < 8; ++w) {
                    const float4 q = sm[w][lane];
                    acc.x += q.x, acc.y += q.y, acc.z += q.z, acc.w += q.w;
                }
                const float f[4] = {acc.x, acc.y, acc.z, acc.w};
                store_scaled(a.dtable + (int64_t)row * a.d + 4 * at, f, a.scale, false);
            }
        }
    }
}

}  // namespace embed
}  // namespace noble
