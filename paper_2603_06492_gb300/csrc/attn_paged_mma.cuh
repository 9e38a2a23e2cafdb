// Attention of a few new tokens over a paged bf16 cache, on warp-wide matrix products.
//
// What bounds it is reading the cache, once; 16 rows (the query heads that share a key
// head, times the new tokens) take part in each product of 16 keys, so that its
// arithmetic stays far below that.  Everything is in registers: a lane loads 16 bytes of
// a key or value row and uses them where they are, because the order of what a product
// sums over, and of its columns, is free as long as both sides agree:
//     S = Q K^T  lane (g, t) = (lane / 4, lane % 4) loads features 32 c + 8 t .. + 7 of
//                key g: the operands of two steps, for which Q has the same order
//     O += P V   lane (g, t) loads features 64 u + 8 g .. + 7 of keys 2t, 2t+1, 2t+8, 2t+9
//                (P's own order) and pairs the keys with byte permutes; column n of
//                step j is feature 64 u + 8 n + j, so a lane ends up with 16
//                consecutive features of two rows
// The warps of a block take turns at its chunk's groups of 16 keys, each with a softmax of
// its own; the four are joined in shared memory at the end.  The next keys load while the
// values' product runs, the next values during the keys'.
//
// 64 sequences up to 32768 tokens, 32 heads on 4 of 128 features: 371 us, 5.6 TB/s.  4 tokens of
// one sequence over 131072: 58 us, 4.7 TB/s.  24 sequences up to 1024 tokens, 16 heads of 64:
// 23 us, of which reading takes 7: two dependent launches, and lengths, pages and keys each wait
// for what is before them.
#pragma once

#include "attn_paged.cuh"
#include "attn_tc.cuh"

namespace noble {
namespace attn {
namespace paged {

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 16 bytes that nothing reads again soon
__device__ __forceinline__ uint4 load16(const __nv_bfloat16 *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}

// Blocks of an SM, which set the registers of a thread: heads of 128 features need all of
// two (253; with three they spill, 64 sequences up to 32768 tokens 552 us for 365).
template <int DP> constexpr int kBlocksPerSm = DP == 64 ? 4 : 2;

// PAGE16: pages of a multiple of 16 tokens, so that a group of 16 keys has one page.
// grid as simt_kernel's
template <int DP, bool PAGE16>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm<DP>) mma_kernel(const __grid_constant__ Args<__nv_bfloat16> a)
{
    constexpr int C = DP / 32, U = DP / 64;
    constexpr int kStep = 64;  // keys of a block at a time
    __shared__ float join_o[4][16][DP + 4], join_m[4][16], join_l[4][16];
    __shared__ int redo[16];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
    const int chunk = blockIdx.x % a.chunks, rb = blockIdx.x / a.chunks, kvh = blockIdx.y, n = blockIdx.z;
    const int group = a.n_q / a.n_kv, rows = group * a.q_len;
    // the page of the first keys, unless a window moves them, while the length is on its way
    const int guess = chunk * a.chunk + 16 * warp, guess_j = guess + (PAGE16 ? 0 : lane & 15);
    const int guessed = guess_j / a.page_size < a.max_pages ? a.page_table[(int64_t)n * a.max_pages + guess_j / a.page_size] : -1;
    const Span sp = span(a, n);
    const Chunks cs = chunks(a, sp);
    if (chunk < cs.first || chunk > cs.last) return;
    const int c0 = chunk * a.chunk, j0 = max(c0, sp.from), j1 = c0 + min(a.chunk, sp.len - c0);

    // rows g and g + 8 of the block: Q, positions, ranges
    uint32_t q[2][C][4];
    int pos[2], hi[2], lo[2];
    float slope[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = rb * kRows + g + 8 * r;
        const bool real = row < rows;
        pos[r] = sp.raw - a.q_len + (real ? row / group : 0);
        hi[r] = real ? min(pos[r] + 1, j1) : 0;
        lo[r] = a.window ? pos[r] - a.window + 1 : 0;
        slope[r] = a.score.slope && real ? a.score.slope[kvh * group + row % group] : 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (real && 32 * c + 8 * t < a.d)
                v = *reinterpret_cast<const uint4 *>(a.q.at((int64_t)n * a.q_len + row / group, kvh * group + row % group) + 32 * c + 8 * t);
            q[r][c][0] = v.x, q[r][c][1] = v.y, q[r][c][2] = v.z, q[r][c][3] = v.w;
        }
    }
    const __nv_bfloat16 *kb = a.k + kvh * a.head, *vb = a.v + kvh * a.head;
    uint4 k[2][C], v[4][U];
    bool bad_page = false;
    // Element offset of a group's first key (PAGE16) or of key lane % 16, -1 where nothing
    // may be read: found a step before its keys load, which would else wait for it.
    int64_t at = 0, at_next;
    auto find = [&](int jb, int known) {
        const int j = jb + (PAGE16 ? 0 : lane & 15);
        const bool in = j < j1 && (PAGE16 || j >= j0);
        at_next = -1;
        if (in) {
            const int id = known >= 0 ? known : a.page_table[(int64_t)n * a.max_pages + j / a.page_size];
            if (id >= 0 && id < a.pages) at_next = id * a.page + j % a.page_size * a.row;
            else bad_page = true;
        }
    };
    auto key = [&](int jb, int e) -> int64_t {  // of key e of a group
        if (PAGE16) return at >= 0 && jb + e >= j0 && jb + e < j1 ? at + e * a.row : -1;
        return __shfl_sync(0xffffffffu, at, e);
    };
    auto load_k = [&](int jb) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t p = key(jb, g + 8 * h);
#pragma unroll
            for (int c = 0; c < C; ++c)
                k[h][c] = p >= 0 && 32 * c + 8 * t < a.d ? load16(kb + p + 32 * c + 8 * t) : make_uint4(0, 0, 0, 0);
        }
    };
    auto load_v = [&](int jb) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t p = key(jb, 2 * t + (e & 1) + 8 * (e >> 1));
#pragma unroll
            for (int u = 0; u < U; ++u)
                v[e][u] = p >= 0 && 64 * u + 8 * g < a.d ? load16(vb + p + 64 * u + 8 * g) : make_uint4(0, 0, 0, 0);
        }
    };

    float o[U][8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) o[u][j][0] = o[u][j][1] = o[u][j][2] = o[u][j][3] = 0.f;

    int jb = (j0 & ~15) + 16 * warp;
    find(jb, jb == guess ? guessed : -1);
    at = at_next;
    load_k(jb);
    load_v(jb);
    find(jb + kStep, -1);
    for (; jb < j1; jb += kStep) {
        // keys without a page count for no row
        const uint32_t ok = PAGE16 ? (at >= 0 ? 0xffffu : 0u) : __ballot_sync(0xffffffffu, at >= 0) & 0xffffu;
        float s[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            s[h][0] = s[h][1] = s[h][2] = s[h][3] = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                mma16816(s[h], q[0][c][0], q[1][c][0], q[0][c][1], q[1][c][1], k[h][c].x, k[h][c].y);
                mma16816(s[h], q[0][c][2], q[1][c][2], q[0][c][3], q[1][c][3], k[h][c].z, k[h][c].w);
            }
        }
        at = at_next;
        load_k(jb + kStep);
        uint32_t p[2][2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float x[4], top = m[r];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int w = 8 * (e >> 1) + 2 * t + (e & 1), j = jb + w;
                float y = s[e >> 1][2 * r + (e & 1)] * a.score.scale;
                if (a.score.softcap > 0.f) y = a.score.softcap * tanh_exp(y / a.score.softcap);
                if (a.score.slope) y -= slope[r] * (float)(pos[r] - j);
                x[e] = j >= lo[r] && j >= j0 && j < hi[r] && (ok >> w & 1) ? y * kLog2e : -INFINITY;
                top = fmaxf(top, x[e]);
            }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const float base = top == -INFINITY ? 0.f : top;
            if (__any_sync(0xffffffffu, top > m[r])) {
                const float f = exp2_fast(m[r] - base);
                l[r] *= f;
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int j = 0; j < 8; ++j) o[u][j][2 * r] *= f, o[u][j][2 * r + 1] *= f;
                m[r] = top;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = exp2_fast(x[e] - base);
            l[r] += (x[0] + x[1]) + (x[2] + x[3]);
            p[r][0] = ptx::pack_bf16x2(x[0], x[1]), p[r][1] = ptx::pack_bf16x2(x[2], x[3]);
        }
        __syncwarp();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint4 w0 = v[0][u], w1 = v[1][u], w2 = v[2][u], w3 = v[3][u];
            const uint32_t v0[4] = {w0.x, w0.y, w0.z, w0.w}, v1[4] = {w1.x, w1.y, w1.z, w1.w}, v2[4] = {w2.x, w2.y, w2.z, w2.w},
                           v3[4] = {w3.x, w3.y, w3.z, w3.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t sel = j & 1 ? 0x7632 : 0x5410;
                mma16816(o[u][j], p[0][0], p[1][0], p[0][1], p[1][1], __byte_perm(v0[j / 2], v1[j / 2], sel),
                         __byte_perm(v2[j / 2], v3[j / 2], sel));
            }
        }
        load_v(jb + kStep);
        find(jb + 2 * kStep, -1);
    }
    if (bad_page) raise_status(a.status, kStatusBadIndex);

    // join the warps: each brings its rows to shared memory, thread (row, eighth) sums
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
        if (t == 0) join_m[warp][g + 8 * r] = m[r], join_l[warp][g + 8 * r] = l[r];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int j = 0; j < 8; j += 4)
                    *reinterpret_cast<float4 *>(&join_o[warp][g + 8 * r][64 * u + 16 * t + 8 * b + j]) =
                        make_float4(o[u][j][2 * r + b], o[u][j + 1][2 * r + b], o[u][j + 2][2 * r + b], o[u][j + 3][2 * r + b]);
    }
    if (threadIdx.x < 16) redo[threadIdx.x] = 0;
    __syncthreads();
    const int r = threadIdx.x / 8, part = threadIdx.x % 8, row = rb * kRows + r;
    if (row < rows) {
        float top = fmaxf(fmaxf(join_m[0][r], join_m[1][r]), fmaxf(join_m[2][r], join_m[3][r]));
        const float base = top == -INFINITY ? 0.f : top;
        float w[4], sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = exp2_fast(join_m[i][r] - base), sum += w[i] * join_l[i][r];
        const int64_t tok = (int64_t)n * a.q_len + row / group;
        const int h = kvh * group + row % group;
        const bool single = cs.first == cs.last;
        const int64_t pt = (tok * a.n_q + h) * a.chunks + chunk;
        const float inv = !single ? 1.f : sum > 0.f ? 1.f / sum : 0.f;
        bool fine = isfinite(sum);
#pragma unroll
        for (int c = 0; c < DP / 32; ++c) {
            const int f = 32 * c + 4 * part;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 y = *reinterpret_cast<const float4 *>(&join_o[i][r][f]);
                x.x = fmaf(w[i], y.x, x.x), x.y = fmaf(w[i], y.y, x.y), x.z = fmaf(w[i], y.z, x.z), x.w = fmaf(w[i], y.w, x.w);
            }
            x.x *= inv, x.y *= inv, x.z *= inv, x.w *= inv;
            fine = fine && isfinite(x.x) && isfinite(x.y) && isfinite(x.z) && isfinite(x.w);
            if (f < a.d) {
                if (single) store4(a.o.at(tok, h) + f, x);
                else *reinterpret_cast<float4 *>(a.part_o + pt * a.d + f) = x;
            }
        }
        if (part == 0) {
            if (!single) a.part_ml[2 * pt] = top * kLn2, a.part_ml[2 * pt + 1] = sum;
            else if (a.lse) a.lse[tok * a.n_q + h] = sum > 0.f ? (top + log2f(sum)) * kLn2 : -INFINITY;
        }
        if (single && !fine) redo[r] = 1;
    }
    __syncthreads();
    for (int i = warp; i < kRows; i += kThreads / 32) {
        const int rr = rb * kRows + i;
        if (redo[i]) row_paged(a, (int64_t)n * a.q_len + rr / group, kvh * group + rr % group, lane);
    }
}

}  // namespace paged
}  // namespace attn
}  // namespace noble
