// The orthogonalising iteration of small matrices (muon.cuh has the mathematics) in one launch: up to
// 128 rows by 2048 columns, a cluster of up to eight blocks per matrix.  15 launches of a few us of
// work each would take their gaps.
//
// X stays in shared memory throughout, each block holding up to 256 of its columns; all matrices in
// pairs (v = hi + lo).  One step:
//   A   each block multiplies its columns (tcgen05, K = its columns) and leaves its part of the sum in
//       shared memory, where the block that owns the rows reads it (distributed shared memory).
//       That one adds the parts up, its own first, in a fixed order and sends its rows of A to all;
//   B = a I + b A + c A A   in every block, in place of A;
//   X <- B X                each block its columns, in place.
// A tile of 128 rows by 64 columns with the 128-byte swizzle is the operand along K of the first
// product and the operand across K of the last one: the descriptors differ, the bytes do not.
// Up to 64 rows, A and B have 64 rows and columns.
//
// What bounds it is the chain of its parts.  (64 x 1024, 1024 x 64, 64 x 64) on eight blocks each: 10300
// cycles a step, of which the three products have 4000 (62 cycles per tcgen05.mma, whether N is 64 or
// 128), the exchange of A 3700, the passes over B and X 2000.  A whole call in a captured graph takes 40 us
// in place of 120 by 15 launches of muon_gemm.cuh; 64 x 64 33 for 86; 128 x 2048 74 for 158.
// Lanes next to each other exchange bytes next to each other: 16 bytes of one row per lane take three
// cycles a lane (sent as columns, 23000 of a step's 36000 cycles).
#pragma once

#include "muon_gemm.cuh"

namespace noble {
namespace muon {
namespace small {

constexpr int kRows = 128, kBlocks = 8, kCols = 256;  // rows of X; blocks of a cluster, columns of a block at most
constexpr int kFewBlocks = 4;                         // at least: all add up parts, with columns or without
constexpr int kThreads = 512;
constexpr uint32_t kTile = kRows * 128;         // 128 rows of 64 columns
constexpr uint32_t kLow = 4 * kTile;            // X: four tiles, and as many of low parts
constexpr uint32_t kPoly = 8 * kTile;           // parts of A in fp32, A, then B: two tiles, two of low parts
constexpr uint32_t kBarOff = kPoly + 4 * kTile;
constexpr uint32_t kBytes = kBarOff + 48, kDynamic = kBytes + 1024;

struct Args {
    Batch b;
    int cols[kMost];  // of a block: a multiple of 64
    int steps;
    uint32_t *status;
};

// A group of eight elements of a tile.
__device__ __forceinline__ uint32_t at(int row, int col) { return (uint32_t)(col / 64) * kTile + row * 128 + ((((col % 64) / 8) ^ (row & 7)) << 4); }

// Into a block of the cluster; a barrier of that block counts the bytes.
__device__ __forceinline__ void remote_store(uint32_t cluster_addr, const uint2 &v, uint32_t cluster_bar)
{
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];" ::"r"(cluster_addr), "r"(v.x),
                 "r"(v.y), "r"(cluster_bar)
                 : "memory");
}

// Eight values as halves; what is left of them stays in f.
__device__ __forceinline__ uint4 halves(float *f)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
        const float2 r = __half22float2(h);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
        f[2 * i] -= r.x, f[2 * i + 1] -= r.y;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// Four values in pairs.
__device__ __forceinline__ uint2 halves(float a, float b, float c, float d, uint2 *lo)
{
    const __half2 h = __floats2half2_rn(a, b), i = __floats2half2_rn(c, d);
    const float2 r = __half22float2(h), s = __half22float2(i);
    *lo = make_uint2(mma::pack_half(a - r.x, b - r.y), mma::pack_half(c - s.x, d - s.y));
    return make_uint2(*reinterpret_cast<const uint32_t *>(&h), *reinterpret_cast<const uint32_t *>(&i));
}
__device__ __forceinline__ void add_eight(const uint4 &q, float scale, float *f)
{
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 r = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
        f[2 * i] = fmaf(scale, r.x, f[2 * i]), f[2 * i + 1] = fmaf(scale, r.y, f[2 * i + 1]);
    }
}

__global__ void __launch_bounds__(kThreads, 1) iterate_kernel(const __grid_constant__ Args g)
{
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = ptx::smem_u32(smem_raw), sbase = (raw + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (sbase - raw);
    const uint32_t bar = sbase + kBarOff, a_bar = bar + 8, meet_bar = bar + 16;  // products; A; blocks (two)
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + kBarOff + 32);
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, quarter = warp % 4, group = warp / 4;
    const uint32_t rank = cluster::ctarank();
    const int blocks = (int)cluster::nctarank();
    const Matrix &M = g.b.t[blockIdx.x / blocks];
    const int cols = g.cols[blockIdx.x / blocks], c0 = (int)rank * cols;
    const int side = M.m <= 64 ? 64 : 128, own = side / blocks;  // of A; rows that a block adds up
    const int holders = (M.k + cols - 1) / cols;                 // blocks that have columns
    const bool holds = (int)rank < holders;

    ptx::griddep_launch();
    if (tid == 0) {
        ptx::mbar_init(bar, 1);
        ptx::mbar_init(a_bar, 1);
        for (int i = 0; i < 2; ++i) ptx::mbar_init(meet_bar + 8 * i, (uint32_t)blocks);
        ptx::fence_barrier_init();
    }
    if (warp == 0) {
        ptx::tmem_alloc(ptx::smem_u32(tmem_slot), 512);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    cluster::sync();  // all blocks' barriers are initialised
    ptx::tc_fence_after();
    const uint32_t tmem = *tmem_slot, lanes = tmem + ((uint32_t)(quarter * 32) << 16);
    // in every epilogue: a thread has this row and a quarter of the columns
    const int row = quarter * 32 + lane;
    const bool rows = quarter * 32 < side;

    ptx::griddep_wait();
    // X: groups of eight columns that have elements, zeros elsewhere
    for (int i = tid; i < kRows * cols / 8; i += kThreads) {
        const int r = i / (cols / 8), c = i % (cols / 8) * 8;
        const bool in = r < M.m && c0 + c < M.k;
        const int64_t e = (int64_t)r * M.ld + c0 + c;
        const uint4 none = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4 *>(smem + at(r, c)) = in ? *reinterpret_cast<const uint4 *>(M.x + e) : none;
        *reinterpret_cast<uint4 *>(smem + kLow + at(r, c)) = in ? *reinterpret_cast<const uint4 *>(M.x_lo + e) : none;
    }

    uint32_t phase = 0;
    bool ok = true;
    // D = P Q^T over `chunks` tiles along K, by one thread: lo hi, hi lo, hi hi; the operands are in
    // place once all threads are here, and D is complete when they are through
    auto multiply = [&](uint32_t d, uint32_t p, uint32_t p_lo, uint32_t q, uint32_t q_lo, int chunks, int n, bool across) {
        ptx::fence_proxy_async_smem();
        ptx::tc_fence_before();
        __syncthreads();
        if (tid == 0 && ok) {
            ptx::tc_fence_after();
            const uint32_t idesc = mma::idesc_f16(kRows, n, across);
            const uint64_t first = ptx::smem_desc_sw128(sbase, across ? kTile : 16, 1024), a_first = ptx::smem_desc_sw128(sbase, 16, 1024);
            const uint32_t b_next = across ? 128 : 2, b_tile = across ? 512 : kTile / 16;  // descriptors count 16 bytes
            uint32_t add = 0;
#pragma unroll 1
            for (int seg = 0; seg < 3; ++seg) {
                uint64_t a = a_first + (seg == 0 ? p_lo : p) / 16, b = first + (seg == 1 ? q_lo : q) / 16;
#pragma unroll 1
                for (int i = 0; i < chunks; ++i, a += kTile / 16, b += b_tile) {
                    ptx::mma_bf16(d, a, b, idesc, add);
                    add = 1;
#pragma unroll
                    for (int k = 1; k < 4; ++k) ptx::mma_bf16(d, a + 2 * k, b + b_next * k, idesc, 1u);
                }
            }
            ptx::mma_commit(bar);
        }
        // a wait that gave up is reported, and given once more for what is in flight
        if (ok && !ptx::mbar_wait(bar, phase, g.status)) {
            ptx::mbar_wait(bar, phase, nullptr);
            ok = false;
        }
        phase ^= 1;
        __syncwarp();
        ptx::tc_fence_after();
    };

    // All blocks have come here, and see what the others wrote to their shared memory.  The one of the two
    // barriers is reached again only after all blocks have left it: A arrives from each in between.
    auto meet = [&](int which, uint32_t parity) {
        __syncthreads();
        if (tid < blocks) cluster::mbar_arrive(cluster::map_to_rank(meet_bar + 8 * which, tid));
        if (ok) ok = ptx::mbar_wait_cluster(meet_bar + 8 * which, parity, g.status);
        __syncwarp();
    };

    for (int step = 0; step < g.steps; ++step) {
        const uint32_t parity = step & 1;
        if (tid == 0) ptx::mbar_arrive_expect_tx(a_bar, (uint32_t)(side * side * 4));
        // ---- A: parts, a row's groups of four elements in an order that keeps lanes of one column on
        // different banks
        const uint32_t parts = kPoly + (side == 64 ? kTile : 0);  // 64 rows leave room beside A
        auto part = [&](int r, int four) { return parts + (uint32_t)(r * side + (four ^ (r & (side / 4 - 1))) * 4) * 4; };
        if (holds) {
            multiply(tmem, 0, kLow, 0, kLow, cols / 64, side, false);
            for (int col0 = side / 4 * group; rows && col0 < side / 4 * (group + 1); col0 += 16) {
                float v[16];
                ptx::tmem_ld_32x32b_x16(lanes + col0, v);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<float4 *>(smem + part(row, col0 / 4 + j)) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
            }
        }
        meet(0, parity);
        // own rows, in groups of four elements; each block begins with itself, so that not one is asked by all
        constexpr int kGroups = kRows * kRows / 4 / kFewBlocks / kThreads;
        const int per_row = side / 4;
        uint2 hi[kGroups], lo[kGroups];
#pragma unroll
        for (int k = 0; k < kGroups; ++k) {
            const int i = tid + kThreads * k;
            if (i >= own * per_row) break;
            const uint32_t from = sbase + part((int)rank * own + i / per_row, i % per_row);
            float4 u[kBlocks];
#pragma unroll
            for (int q = 0; q < kBlocks; ++q) {
                const int p = ((int)rank + q) & (blocks - 1);
                u[q] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (q < blocks && p < holders) u[q] = cluster::ld4(cluster::map_to_rank(from, p));
            }
#pragma unroll
            for (int q = 1; q < kBlocks; ++q) u[0].x += u[q].x, u[0].y += u[q].y, u[0].z += u[q].z, u[0].w += u[q].w;
            constexpr float f = kScaleA / (kScaleX * kScaleX);
            hi[k] = halves(u[0].x * f, u[0].y * f, u[0].z * f, u[0].w * f, &lo[k]);
        }
        if (side != 64) meet(1, parity);  // all parts are read
#pragma unroll
        for (int k = 0; k < kGroups; ++k) {
            const int i = tid + kThreads * k, r = (int)rank * own + i / per_row, col = i % per_row * 4;
            if (i >= own * per_row) break;
            const uint32_t to = sbase + kPoly + at(r, col) + col % 8 * 2;
#pragma unroll
            for (int q = 0; q < kBlocks; ++q) {
                const int p = ((int)rank + q) & (blocks - 1);
                if (q >= blocks) continue;
                const uint32_t there = cluster::map_to_rank(a_bar, p);
                remote_store(cluster::map_to_rank(to, p), hi[k], there);
                remote_store(cluster::map_to_rank(to + 2 * kTile, p), lo[k], there);
            }
        }
        if (ok) ok = ptx::mbar_wait_cluster(a_bar, parity, g.status);
        __syncwarp();
        if (!holds) continue;
        // ---- B
        multiply(tmem, kPoly, kPoly + 2 * kTile, kPoly, kPoly + 2 * kTile, side / 64, side, false);
        for (int col0 = side / 4 * group; rows && col0 < side / 4 * (group + 1); col0 += 16) {
            float v[16];
            ptx::tmem_ld_32x32b_x16(lanes + col0, v);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float *f = v + 8 * q;
                uint4 *h = reinterpret_cast<uint4 *>(smem + kPoly + at(row, col0 + 8 * q));
                uint4 *l = reinterpret_cast<uint4 *>(smem + kPoly + 2 * kTile + at(row, col0 + 8 * q));
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    f[j] *= muon::kC * kScaleB / (kScaleA * kScaleA);
                    if (row == col0 + 8 * q + j) f[j] += muon::kA * kScaleB;
                }
                add_eight(*h, muon::kB * kScaleB / kScaleA, f);
                add_eight(*l, muon::kB * kScaleB / kScaleA, f);
                *h = halves(f);
                *l = halves(f);
            }
        }
        // ---- X
        multiply(tmem + 128, kPoly, kPoly + 2 * kTile, 0, kLow, side / 64, cols, true);
        for (int col0 = cols / 4 * group; rows && col0 < cols / 4 * (group + 1); col0 += 16) {
            float v[16];
            ptx::tmem_ld_32x32b_x16(lanes + 128 + col0, v);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float *f = v + 8 * q;
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] *= 1.f / kScaleB;
                *reinterpret_cast<uint4 *>(smem + at(row, col0 + 8 * q)) = halves(f);
                *reinterpret_cast<uint4 *>(smem + kLow + at(row, col0 + 8 * q)) = halves(f);
            }
        }
    }
    __syncthreads();
    __half *o = const_cast<__half *>(M.o), *o_lo = const_cast<__half *>(M.o_lo);
    for (int i = tid; i < M.m * (cols / 8); i += kThreads) {
        const int r = i / (cols / 8), c = i % (cols / 8) * 8;
        if (c0 + c >= M.k) continue;
        const int64_t e = (int64_t)r * M.ld + c0 + c;
        *reinterpret_cast<uint4 *>(o + e) = *reinterpret_cast<const uint4 *>(smem + at(r, c));
        *reinterpret_cast<uint4 *>(o_lo + e) = *reinterpret_cast<const uint4 *>(smem + kLow + at(r, c));
    }
    ptx::tc_fence_before();
    __syncthreads();
    cluster::sync();  // no block leaves while others may still write to it
    if (warp == 0) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, 512);
    }
}

}  // namespace small
}  // namespace muon
}  // namespace noble
