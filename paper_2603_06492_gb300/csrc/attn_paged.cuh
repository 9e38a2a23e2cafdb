// Attention of a few new tokens per sequence over a paged cache.
//
// Bound by reading the cache.  The query heads that share a key head, and the new tokens
// of a sequence, are the rows of one block (16 of them), so that a key is read for all of
// them at once; each further 16 rows are a block that reads the keys again (16 sequences up to
// 16380 tokens, 32 heads on 4 of 128, bf16: 1 new token 71 us, 2 76, 4 120, 8 200).  The keys of a sequence are split into chunks, a
// block each, since a batch alone has too few sequences to load 152 SMs; a second
// kernel joins the chunks' results by their maxima and sums, in order.  fp32
// works out all 16 rows whatever is real and loads nothing during a product: 24 sequences up to
// 1000 tokens, 16 heads of 64, one row each: 73 us, 1.4 TB/s.
#pragma once

#include "attn_simt.cuh"
#include "sm100_ptx.cuh"

namespace noble {
namespace attn {
namespace paged {

constexpr int kRows = 16, kKeys = 64, kThreads = 128;
// Tokens of a sequence: the positions that a block works out beyond its last key, a step or two of
// 64, stay within 32 bits.
constexpr int kMaxLen = INT32_MAX - 65535;

template <typename T>
struct Args {
    Heads<const T> q;
    Heads<T> o;
    const T *k, *v;
    const int32_t *page_table, *kv_len;
    float *lse;                // [rows][n_q] or NULL
    float *part_o, *part_ml;   // [n_seq * n_kv][rows of a sequence][chunks][d], ... [2]
    int64_t page, row, head;   // strides of the cache
    int64_t max_pages, max_len;
    int pages, page_size, n_seq, q_len, n_q, n_kv, d, window;
    int chunk, chunks;         // keys of a chunk (a multiple of kKeys), chunks of a sequence
    Score score;
    uint32_t *status;
};

// What the tokens of sequence n see of its cache: its first `len` tokens (all `raw`
// of them, if that is no error) but the first `from`, which are outside every window.
struct Span {
    int raw, len, from;
};
template <typename T>
__device__ __forceinline__ Span span(const Args<T> &a, int n)
{
    const int64_t most = min((int64_t)a.max_pages * a.page_size, a.max_len);
    const int raw = max(a.kv_len[n], 0);
    const int len = raw > most ? (int)most : raw;
    if (raw > most) raise_status(a.status, kStatusBadIndex);
    const int first = raw - a.q_len;  // the first new token's position
    return {raw, len, a.window && first - a.window + 1 > 0 ? min(first - a.window + 1, len) : 0};
}

// The chunks with keys that sequence n sees, one at least, which also writes what a sequence
// without such keys gets: a window behind a length that was cut leaves none.
struct Chunks {
    int first, last;
};
template <typename T>
__device__ __forceinline__ Chunks chunks(const Args<T> &a, const Span &sp)
{
    const int last = max(sp.len - 1, 0) / a.chunk;
    return {min(sp.from / a.chunk, last), last};
}

// Place of the key at position j, or -1 if its page is not one of the cache's.
template <typename T>
__device__ __forceinline__ int64_t place(const Args<T> &a, int n, int j)
{
    const int id = a.page_table[(int64_t)n * a.max_pages + j / a.page_size];
    return id < 0 || id >= a.pages ? -1 : id * a.page + j % a.page_size * a.row;
}

// One row by one warp over exactly the keys that it sees (see row_fwd).
template <typename T>
__device__ __noinline__ void row_paged(const Args<T> &a, int64_t t, int h, int lane)
{
    count_row(lane);
    const int n = (int)(t / a.q_len), g = h / (a.n_q / a.n_kv);
    const Span sp = span(a, n);
    const int pos = sp.raw - a.q_len + (int)(t % a.q_len);
    float q[4], acc[4] = {}, m = -INFINITY, l = 0.f;
    row_load(q, a.q.at(t, h), a.d, lane);
    for (int j = a.window ? max(0, pos - a.window + 1) : 0; j < min(pos + 1, sp.len); ++j) {
        const int64_t at = place(a, n, j);
        if (at < 0) continue;
        float x[4];
        row_load(x, a.k + at + g * a.head, a.d, lane);
        const float s = row_score(a.score, row_dot(q, x), h, pos, j, nullptr);
        row_load(x, a.v + at + g * a.head, a.d, lane);
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
    row_store(a.o.at(t, h), acc, a.d, lane);
    if (a.lse && lane == 0) a.lse[t * a.n_q + h] = l == 0.f ? -INFINITY : m + logf(l);
}

// grid: x = chunk + chunks * block of rows, y = key head, z = sequence
template <int DP, typename T>
__global__ void __launch_bounds__(kThreads) simt_kernel(const __grid_constant__ Args<T> a)
{
    constexpr int R = 2, RS = 8;
    extern __shared__ float sm[];
    float *Q = sm, *KV = Q + kRows * simt::kLd<DP>, *P = KV + kKeys * simt::kLd<DP>;
    __shared__ int64_t at[kKeys];
    __shared__ int redo[kRows];
    const int tid = threadIdx.x, tx = tid % 16, ty = tid / 16;
    const int chunk = blockIdx.x % a.chunks, rb = blockIdx.x / a.chunks, g = blockIdx.y, n = blockIdx.z;
    const int group = a.n_q / a.n_kv, rows = group * a.q_len;
    const Span sp = span(a, n);
    const int raw = sp.raw, c0 = chunk * a.chunk, j0 = max(c0, sp.from), j1 = c0 + min(a.chunk, sp.len - c0);
    const Chunks cs = chunks(a, sp);
    if (chunk < cs.first || chunk > cs.last) return;
    // row r: token r / group, head g * group + r % group
    float m[R], l[R], slope[R];
    int hi[R], lo[R];
    float4 acc[R][DP / 64];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = rb * kRows + ty + RS * r;
        const int pos = raw - a.q_len + row / group;
        hi[r] = row < rows ? min(pos + 1, sp.len) : 0;
        lo[r] = a.window ? pos - a.window + 1 : 0;
        slope[r] = a.score.slope && row < rows ? a.score.slope[g * group + row % group] : 0.f;
        m[r] = -INFINITY, l[r] = 0.f;
#pragma unroll
        for (int u = 0; u < DP / 64; ++u) acc[r][u] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (int c = tid; c < kRows * DP / 4; c += kThreads) {
        const int rr = c / (DP / 4), f = c % (DP / 4) * 4, row = rb * kRows + rr;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row < rows && f < a.d) v = load4(a.q.at((int64_t)n * a.q_len + row / group, g * group + row % group) + f);
        *reinterpret_cast<float4 *>(Q + rr * simt::kLd<DP> + f) = v;
    }
    auto load = [&](const T *base) {
        for (int c = tid; c < kKeys * DP / 4; c += kThreads) {
            const int key = c / (DP / 4), f = c % (DP / 4) * 4;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (at[key] >= 0 && f < a.d) v = load4(base + at[key] + g * a.head + f);
            *reinterpret_cast<float4 *>(KV + key * simt::kLd<DP> + f) = v;
        }
    };
    for (int jb = j0; jb < j1; jb += kKeys) {
        __syncthreads();
        if (tid < kKeys) {
            at[tid] = jb + tid < j1 ? place(a, n, jb + tid) : -1;
            if (jb + tid < j1 && at[tid] < 0) raise_status(a.status, kStatusBadIndex);
        }
        __syncthreads();
        load(a.k);
        __syncthreads();
        float s[R][4];
        simt::dots<DP, R, RS>(s, Q, KV, ty, tx);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int pos = raw - a.q_len + (rb * kRows + ty + RS * r) / group;
            float top = m[r];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int j = jb + tx + 16 * c;
                s[r][c] = j >= lo[r] && j < min(hi[r], j1) && at[tx + 16 * c] >= 0
                              ? simt::score(a.score, slope[r], s[r][c], pos - j, nullptr) : -INFINITY;
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
                P[(ty + RS * r) * simt::kPP + tx + 16 * c] = s[r][c];
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
        load(a.v);
        __syncthreads();
        simt::accumulate<DP, R, RS>(acc, P, KV, ty, tx);
    }
    if (tid < kRows) redo[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = rb * kRows + ty + RS * r;
        if (row >= rows) continue;
        const int64_t t = (int64_t)n * a.q_len + row / group;
        const int h = g * group + row % group;
        if (cs.first == cs.last) {
            if (!simt::finite(acc[r]) || !isfinite(l[r])) redo[ty + RS * r] = 1;
            simt::store_row(a.o.at(t, h), acc[r], l[r] > 0.f ? 1.f / l[r] : 0.f, a.d, tx);
            if (a.lse && tx == 0) a.lse[t * a.n_q + h] = l[r] > 0.f ? m[r] + logf(l[r]) : -INFINITY;
        } else {
            const int64_t p = (t * a.n_q + h) * a.chunks + chunk;
            simt::store_row(a.part_o + p * a.d, acc[r], 1.f, a.d, tx);
            if (tx == 0) a.part_ml[2 * p] = m[r], a.part_ml[2 * p + 1] = l[r];
        }
    }
    __syncthreads();
    for (int r = tid / 32; r < kRows; r += kThreads / 32) {
        const int row = rb * kRows + r;
        if (redo[r]) row_paged(a, (int64_t)n * a.q_len + row / group, g * group + row % group, tid % 32);
    }
}

// The chunks' results of a row, each scaled to the common maximum: `per_row` warps of the
// block's eight (a power of two) take every per_row-th chunk, the first adds theirs up.
template <typename T>
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ Args<T> a, int per_row)
{
    __shared__ float4 sum_o[8][32];
    __shared__ float sum_l[8];
    ptx::griddep_wait();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, part = warp % per_row;
    const int64_t u = (int64_t)blockIdx.x * (8 / per_row) + warp / per_row, rows = (int64_t)a.n_seq * a.q_len * a.n_q;
    const int64_t t = u / a.n_q;
    const int h = (int)(u % a.n_q);
    int c0 = 0, c1 = -1;
    if (u < rows) {
        const Chunks cs = chunks(a, span(a, (int)(t / a.q_len)));
        c0 = cs.first, c1 = cs.last;
    }
    const bool work = c1 > c0;  // a single chunk has written the result itself
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f, m = -INFINITY;
    if (work) {
        for (int c = c0 + lane; c <= c1; c += 32) m = fmaxf(m, a.part_ml[2 * (u * a.chunks + c)]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float base = m == -INFINITY ? 0.f : m;
#pragma unroll 8
        for (int c = c0 + part; c <= c1; c += per_row) {
            const int64_t p = u * a.chunks + c;
            const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + 2 * p);
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (4 * lane < a.d) x = load4(a.part_o + p * a.d + 4 * lane);
            const float w = exp2f((ml.x - base) * kLog2e);
            l = fmaf(w, ml.y, l);
            acc.x = fmaf(w, x.x, acc.x), acc.y = fmaf(w, x.y, acc.y), acc.z = fmaf(w, x.z, acc.z), acc.w = fmaf(w, x.w, acc.w);
        }
    }
    sum_o[warp][lane] = acc;
    if (lane == 0) sum_l[warp] = l;
    __syncthreads();
    if (!work || part) return;
    for (int i = 1; i < per_row; ++i) {
        const float4 x = sum_o[warp + i][lane];
        acc.x += x.x, acc.y += x.y, acc.z += x.z, acc.w += x.w;
        l += sum_l[warp + i];
    }
    const bool ok = isfinite(acc.x) && isfinite(acc.y) && isfinite(acc.z) && isfinite(acc.w) && isfinite(l);
    if (!__all_sync(0xffffffffu, ok)) {
        row_paged(a, t, h, lane);
        return;
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    if (4 * lane < a.d) store4(a.o.at(t, h) + 4 * lane, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
    if (a.lse && lane == 0) a.lse[u] = l > 0.f ? m + logf(l) : -INFINITY;
}

}  // namespace paged
}  // namespace attn
}  // namespace noble
