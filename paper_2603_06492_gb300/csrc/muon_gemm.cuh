// The products of the orthogonalising iteration on the tensor cores (muon.cuh has the
// mathematics), for all matrices of a group in one launch:
//
//   C = alpha P Q^T + beta D + diag I       P [m][k], Q [n][k] or, for X <- B X, stored [k][n]
//
// fp16 operands, fp32 accumulation in TMEM, fp16 results.  A matrix in pairs (v = hi + lo)
// takes three segments of K into one accumulator: lo hi, hi lo, hi hi.  The large terms come last, as every
// add to an accumulator costs it half a bit of fp32 (64 x 64 with hi hi first: X 4e-6 off).
//
// CTA pairs as in tc_pair.cuh: tiles of 256 x bn, TMA -> ring of six stages -> tcgen05.mma by
// the leader's warp 1 -> TMEM -> eight epilogue warps per CTA, two accumulators in turn.
// Units of work are given to the pairs in turn, the longest first, there and back: what a round
// leaves over goes to the pairs that had the shortest units in the one before.
//  - A and A A are symmetric: tiles that lie below the diagonal are not computed, the others
//    are also stored transposed.  (2048 x 8192: 72 units in place of 128 for X X^T.)
//  - A product of few tiles and long K is split along K.  Each warp stores its part of the
//    accumulator, 32 columns at a time; the last of a tile's splits to arrive there, known by a
//    counter, adds all of them up in order, so that no sum depends on who is last, and
//    nobody waits.
#pragma once

#include "muon.cuh"
#include "tc_pair.cuh"

namespace noble {
namespace muon {
namespace mma {

constexpr int kRows = 256;  // of a tile: 128 in each CTA of the pair
constexpr int kBK = 64;
// Bytes of operands in flight hide the latency of L2: six stages of tiles of 256 columns, or eight
// of 128 (2048 x 2048 by itself, 72 units of 32 k-blocks: 8.5 us a unit with six).
constexpr int kStagesWide = 6, kStagesNarrow = 8;
constexpr int kPairs = 76;  // of a GB300; a constant, as the splits set the order of sums
constexpr int kMostSplits = 16;

struct Problem {
    int m, n;          // of C
    int kb, segs;      // k-blocks of a segment; segments: 1, or 3 for pairs
    int bn;            // columns of a tile: 128 or 256
    int tiles_m, tiles_n;
    int sym, b_mn;
    int nsplit, kb_per_split;
    int unit_begin;    // first of the launch: unit = tile * nsplit + split
    float alpha, beta, diag;
    const __half *d, *d_lo;
    int ldd;           // elements between rows of D, a multiple of 8
    int pairs;         // C has low parts
    // k-blocks that are added up in TMEM before the next ones get columns of their own: the tensor core
    // cuts what it adds to an accumulator off to fp32, so that a long sum of like terms (the diagonal of
    // X X^T) comes out too small, by 2^-24 for each of its adds
    int piece_kb;
    float *part;       // [unit][256][bn] as the warps hold them
    uint32_t *count;   // [tile][2 CTAs][8 warps][4 chunks], zero before and after
};
// N: matrices at most; a launch's arguments are copied to the GPU, so that few take less.
template <int N>
struct Args {
    CUtensorMap map[N][6];  // P, P low, Q, Q low, C, C low
    Problem p[N];
    int n, units;
    uint32_t *status;
};

template <bool WIDE>
struct Smem {
    static constexpr int kStages = WIDE ? kStagesWide : kStagesNarrow;
    static constexpr uint32_t kA = 128 * kBK * 2, kStage = kA + (WIDE ? 128 : 64) * kBK * 2;
    static constexpr uint32_t kStgOff = kStages * kStage;  // 4 KB per epilogue warp
    static constexpr uint32_t kBarOff = kStgOff + 8 * 4096;
    static constexpr uint32_t kNumBars = 2 * kStages + 5;  // full, empty, tfull[2], tempty[2], done
    static constexpr uint32_t kBytes = kBarOff + 8 * kNumBars + 16;
    static constexpr uint32_t kDynamic = kBytes + 1024;
};

// Unit u's pair, and a pair's unit in round r.
__host__ __device__ inline int pair_of(int u, int pairs) { return u / pairs % 2 ? pairs - 1 - u % pairs : u % pairs; }
__device__ __forceinline__ int unit_of(int r, int pair, int pairs) { return r * pairs + (r % 2 ? pairs - 1 - pair : pair); }

struct Unit {
    int prob, tile, split;
    int m0, n0;  // the tile's first row and column
    int kb_begin, kb_end;
    bool mirror;  // also stored transposed
};

// First tile of row block mp of a symmetric C: those before it keep at or above the diagonal.
__host__ __device__ inline int sym_tiles_before(int mp, int tiles_n, int per) { return mp * tiles_n - per * (mp * (mp - 1) / 2); }

template <int N>
__device__ __forceinline__ Unit locate(const Args<N> &g, int u)
{
    int j = 0;
#pragma unroll 1
    while (j + 1 < g.n && u >= g.p[j + 1].unit_begin) ++j;
    const Problem &P = g.p[j];
    Unit r;
    r.prob = j;
    const int local = u - P.unit_begin;
    r.tile = local / P.nsplit;
    r.split = local - r.tile * P.nsplit;
    int mp, nt;
    if (P.sym) {
        const int per = kRows / P.bn;
        mp = 0;
#pragma unroll 1
        while (mp + 1 < P.tiles_m && r.tile >= sym_tiles_before(mp + 1, P.tiles_n, per)) ++mp;
        nt = mp * per + r.tile - sym_tiles_before(mp, P.tiles_n, per);
        r.mirror = nt * P.bn >= (mp + 1) * kRows;
    } else {
        // groups of eight row blocks, the columns running fastest inside a group
        constexpr int G = 8;
        const int group = r.tile / (G * P.tiles_n), gm = min(G, P.tiles_m - group * G);
        const int in = r.tile - group * G * P.tiles_n;
        mp = group * G + in % gm;
        nt = in / gm;
        r.mirror = false;
    }
    r.m0 = mp * kRows, r.n0 = nt * P.bn;
    r.kb_begin = r.split * P.kb_per_split;
    r.kb_end = min(P.kb * P.segs, r.kb_begin + P.kb_per_split);
    return r;
}

// kind::f16 with fp16 operands and fp32 sums
__device__ __forceinline__ uint32_t idesc_f16(int m, int n, bool b_mn)
{
    return (1u << 4) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

__device__ __forceinline__ uint32_t pack_half(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// WIDE: some tiles have 256 columns.
template <int N, bool WIDE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(tc::pair::kPairThreads, 1)
product_pairs(const __grid_constant__ Args<N> g)
{
    using namespace tc;
    using Smem = mma::Smem<WIDE>;
    constexpr int kStages = Smem::kStages;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = ptx::smem_u32(smem_raw);
    const uint32_t sbase = (raw + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (sbase - raw);
    const uint32_t bar0 = sbase + Smem::kBarOff;
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (kStages + s); };
    auto tfull_bar = [&](int b) { return bar0 + 8u * (2 * kStages + b); };
    auto tempty_bar = [&](int b) { return bar0 + 8u * (2 * kStages + 2 + b); };
    const uint32_t done_bar = bar0 + 8u * (2 * kStages + 4);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + Smem::kBarOff + 8 * Smem::kNumBars);

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = cluster::ctarank();
    const bool leader = rank == 0;
    const int pairs = gridDim.x / 2, first = blockIdx.x / 2;

    if (warp == 0 && lane == 0) {
        ptx::griddep_launch();
        for (int i = 0; i < 6; ++i) ptx::tma_prefetch_desc(&g.map[locate(g, first).prob][i]);
        for (int s = 0; s < kStages; ++s) {
            ptx::mbar_init(full_bar(s), 1);
            ptx::mbar_init(empty_bar(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            ptx::mbar_init(tfull_bar(b), 1);
            ptx::mbar_init(tempty_bar(b), 16);  // 8 epilogue warps in each CTA of the pair
        }
        ptx::mbar_init(done_bar, 1);
        ptx::fence_barrier_init();
    }
    if (warp == 1) {
        pair::tmem_alloc2(ptx::smem_u32(tmem_slot), 512);
        pair::tmem_relinquish2();
    }
    ptx::tc_fence_before();
    __syncthreads();
    cluster::sync();  // the peer's barriers are initialised before any remote use
    ptx::tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp == 0) {
        if (lane == 0) {
            // ---------------- producer (both CTAs)
            ptx::griddep_wait();  // all operands come from earlier kernels of the call
            uint32_t it = 0;
            int s = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (int r = 0, u; ok && (u = unit_of(r, first, pairs)) < g.units; ++r) {
                const Unit t = locate(g, u);
                const Problem &P = g.p[t.prob];
                const int kb_of_seg = P.kb, bh = P.bn / 2, b_mn = P.b_mn;
                const int m0 = t.m0 + 128 * (int)rank, n0 = t.n0 + bh * (int)rank;
                const uint32_t bytes = Smem::kA + (uint32_t)bh * kBK * 2;
                int seg = t.kb_begin / kb_of_seg, kb = t.kb_begin - seg * kb_of_seg;
                seg += 3 - P.segs;  // the last one is hi hi
                for (int i = t.kb_begin; i < t.kb_end; ++i, ++it) {
                    if (!ptx::mbar_wait(empty_bar(s), ph ^ 1, g.status)) {
                        ok = false;
                        break;
                    }
                    const uint32_t fb = cluster::map_to_rank(full_bar(s), 0);
                    if (leader) ptx::mbar_arrive_expect_tx(full_bar(s), 2 * bytes);
                    const uint32_t sA = sbase + s * Smem::kStage, sB = sA + Smem::kA;
                    const CUtensorMap *mP = &g.map[t.prob][seg == 0 ? 1 : 0], *mQ = &g.map[t.prob][seg == 1 ? 3 : 2];
                    const int k = kb * kBK;
                    pair::tma_load_2d_pair(sA, mP, fb, k, m0);
                    if (b_mn)
                        pair::tma_load_4d_pair(sB, mQ, fb, n0 / 64, k / 8);
                    else
                        pair::tma_load_2d_pair(sB, mQ, fb, k, n0);
                    if (++kb == kb_of_seg) kb = 0, ++seg;
                    if (++s == kStages) s = 0, ph ^= 1;
                }
            }
            // the leader's barriers count the peer's bytes too: once they complete, no copy of
            // either CTA is still landing
            if (leader)
                for (uint32_t i = it > (uint32_t)kStages ? it - kStages : 0; i < it; ++i)
                    ptx::mbar_wait(full_bar(i % kStages), (i / kStages) & 1, nullptr);
        }
    } else if (warp == 1) {
        if (lane == 0 && leader) {
            // ---------------- MMA issuer: two stages at a time, descriptors by addition (tc_group.cuh)
            constexpr uint32_t kUnits = Smem::kStage / 16;
            uint32_t *const status = g.status;
            int s = 0, acc = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (int u; ok && (u = unit_of(acc, first, pairs)) < g.units; ++acc) {
                const Unit t = locate(g, u);
                const Problem &P = g.p[t.prob];
                const bool b_mn = P.b_mn != 0;
                const uint32_t idesc = idesc_f16(kRows, P.bn, b_mn);
                const uint64_t a0 = ptx::smem_desc_sw128(sbase, 16, 1024);
                const uint32_t nch = (uint32_t)P.bn / 128;  // chunks of 64 columns in a CTA
                const uint64_t b0 = b_mn ? ptx::smem_desc_sw128(sbase + Smem::kA, 1024, 1024 * nch)
                                         : ptx::smem_desc_sw128(sbase + Smem::kA, 16, 1024);
                const uint32_t stepB = b_mn ? 128u * nch : 2u;
                const int nkb = t.kb_end - t.kb_begin, b = acc & 1, piece = P.piece_kb, bn = P.bn;
                if (!ptx::mbar_wait(tempty_bar(b), ((uint32_t)(acc >> 1) & 1u) ^ 1u, status)) break;
                ptx::tc_fence_after();
                uint32_t d_tmem = tmem + b * 256;
                int next = piece;  // k-block that begins the next piece; pieces are even
                uint32_t add = 0;
                for (int i = 0; i < nkb; i += 2) {
                    if (i == next) d_tmem += bn, next += piece, add = 0;
                    const bool two = i + 1 < nkb;
                    int s2 = s + 1;
                    uint32_t ph2 = ph;
                    if (s2 == kStages) s2 = 0, ph2 ^= 1;
                    if (!ptx::mbar_wait(full_bar(s), ph, status) || (two && !ptx::mbar_wait(full_bar(s2), ph2, status))) {
                        ok = false;
                        break;
                    }
                    const uint64_t so = (uint64_t)((uint32_t)s * kUnits);
                    pair::mma2_bf16(d_tmem, a0 + so, b0 + so, idesc, add);
                    add = 1;
#pragma unroll
                    for (int kk = 1; kk < kBK / 16; ++kk)
                        pair::mma2_bf16(d_tmem, a0 + so + kk * 2, b0 + so + kk * stepB, idesc, 1u);
                    pair::mma2_commit_mc(empty_bar(s), 0x3);
                    if (two) {
                        const uint64_t so2 = (uint64_t)((uint32_t)s2 * kUnits);
#pragma unroll
                        for (int kk = 0; kk < kBK / 16; ++kk)
                            pair::mma2_bf16(d_tmem, a0 + so2 + kk * 2, b0 + so2 + kk * stepB, idesc, 1u);
                        pair::mma2_commit_mc(empty_bar(s2), 0x3);
                        s = s2 + 1, ph = ph2;
                        if (s == kStages) s = 0, ph ^= 1;
                    } else {
                        s = s2, ph = ph2;
                    }
                }
                pair::mma2_commit_mc(tfull_bar(b), 0x3);
            }
            pair::mma2_commit_mc(done_bar, 0x1);
            ptx::mbar_wait(done_bar, 0, nullptr);
        }
    } else {
        // ---------------- epilogue (both CTAs): 32 rows of the accumulator, alternate 32 columns
        const int quarter = warp % 4, half = (warp - 2) / 4, w8 = warp - 2;
        const uint32_t leader_tempty0 = cluster::map_to_rank(tempty_bar(0), 0);
        const uint32_t leader_tempty1 = cluster::map_to_rank(tempty_bar(1), 0);
        const uint32_t stg = sbase + Smem::kStgOff + (uint32_t)w8 * 4096u;
        uint8_t *stg_ptr = smem + Smem::kStgOff + w8 * 4096;
        ptx::griddep_wait();  // parts, counters and D are earlier kernels'
        int acc = 0;
        for (int u; (u = unit_of(acc, first, pairs)) < g.units; ++acc) {
            const Unit t = locate(g, u);
            const Problem &P = g.p[t.prob];
            const int b = acc & 1;
            const int row0 = t.m0 + 128 * (int)rank + 32 * quarter, chunks = P.bn / 64, row = row0 + lane;
            const bool rows_in = row0 < P.m, lows = P.pairs != 0;
            // chunk c in the order of this split: each ends with another one, so that not one of them
            // is the last for all
            auto chunk = [&](int i) { return (i + t.split) & (chunks - 1); };
            auto column = [&](int c) { return t.n0 + 32 * half + 64 * c; };
            // D of a chunk, on its way a chunk ahead
            uint4 d[4], dl[4];
            auto fetch = [&](int i) {
                const int col0 = column(chunk(i));
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    d[q] = dl[q] = make_uint4(0, 0, 0, 0);
                    if (P.d && i < chunks && row < P.m && col0 + 8 * q < P.n) {
                        const int64_t e = (int64_t)row * P.ldd + col0 + 8 * q;
                        d[q] = __ldcg(reinterpret_cast<const uint4 *>(P.d + e));
                        if (lows) dl[q] = __ldcg(reinterpret_cast<const uint4 *>(P.d_lo + e));
                    }
                }
            };
            fetch(0);
            bool ok = ptx::mbar_wait(tfull_bar(b), (uint32_t)(acc >> 1) & 1u, g.status);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            ptx::tc_fence_after();
            const uint32_t lane_addr = tmem + b * 256 + ((uint32_t)(quarter * 32) << 16) + 32 * half;
            // parts[tile][split][CTA][warp][chunk][column][lane]
            const int64_t split_stride = (int64_t)kRows * P.bn;
            float *parts = P.part + (int64_t)t.tile * P.nsplit * split_stride + ((int)rank * 8 + w8) * chunks * 1024 + lane;
            uint32_t *count = P.count + ((t.tile * 2 + (int)rank) * 8 + w8) * 4;
            const bool split = P.nsplit > 1;
            const int pieces = (t.kb_end - t.kb_begin + P.piece_kb - 1) / P.piece_kb;
            // 32 columns of the accumulator: its pieces in order
            auto load = [&](int c, float (&v)[32]) {
                ptx::tmem_ld_32x32b_x32(lane_addr + 64 * c, v);
                for (int k = 1; k < pieces; ++k) {
                    float w[32];
                    ptx::tmem_ld_32x32b_x32(lane_addr + 64 * c + k * P.bn, w);
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] += w[j];
                }
            };
            if (split && rows_in) {
                for (int c = 0; c < chunks && column(c) < P.n; ++c) {
                    float v[32];
                    load(c, v);
                    float *mine = parts + t.split * split_stride + c * 1024;
#pragma unroll
                    for (int j = 0; j < 32; ++j) __stcg(mine + 32 * j, v[j]);
                }
                __threadfence();
            }
            for (int i = 0; rows_in && i < chunks; ++i) {
                const int c = chunk(i), col0 = column(c);
                if (col0 >= P.n) {
                    fetch(i + 1);
                    continue;
                }
                if (split) {
                    uint32_t got = 0;
                    __syncwarp();
                    if (lane == 0) got = atomicAdd(count + c, 1u);
                    got = __shfl_sync(0xffffffffu, got, 0);
                    if (got != (uint32_t)P.nsplit - 1) {
                        fetch(i + 1);
                        continue;
                    }
                    if (lane == 0) count[c] = 0;
                    __threadfence();
                }
                __syncwarp();  // TMEM loads take the whole warp
                float v[32];
                if (split) {
                    // all parts in order, three on their way at first, then two
                    const float *p = parts + c * 1024;
                    auto part = [&](int z, float (&w)[32]) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) w[j] = z < P.nsplit ? __ldcg(p + z * split_stride + 32 * j) : 0.f;
                    };
                    part(0, v);
#pragma unroll 1
                    for (int z = 1; z < P.nsplit; z += 2) {
                        float w[2][32];
                        part(z, w[0]);
                        part(z + 1, w[1]);
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = v[j] + w[0][j] + w[1][j];
                    }
                } else {
                    load(c, v);
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] *= P.alpha;
                if (P.d) {
                    auto add = [&](const uint4 &x, int q) {
                        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[j]));
                            v[8 * q + 2 * j] = fmaf(P.beta, f.x, v[8 * q + 2 * j]);
                            v[8 * q + 2 * j + 1] = fmaf(P.beta, f.y, v[8 * q + 2 * j + 1]);
                        }
                    };
#pragma unroll
                    for (int q = 0; q < 4; ++q) add(d[q], q);
                    if (lows)
#pragma unroll
                        for (int q = 0; q < 4; ++q) add(dl[q], q);
                }
                fetch(i + 1);
                if (P.diag != 0.f && row >= col0 && row < col0 + 32) {
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (row == col0 + j) v[j] += P.diag;
                }
                // 32 x 32 boxes of C, and of it transposed, by TMA: a warp's own stores of them would
                // delay the arrival that hands the accumulator back until they are through
                auto store = [&](const CUtensorMap *map, bool more) {
                    uint32_t h[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) h[j] = pack_half(v[2 * j], v[2 * j + 1]);
                    if (lane == 0) ptx::bulk_wait_read_all();
                    __syncwarp();
                    // rows of 64 bytes in the 64-byte swizzle
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *reinterpret_cast<uint4 *>(stg_ptr + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4)) =
                            make_uint4(h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]);
                    if (t.mirror) {
                        // two rows' elements of a column side by side: an even lane the even column's, an odd
                        // lane the odd column's
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const uint32_t other = __shfl_xor_sync(0xffffffffu, h[j], 1);
                            *reinterpret_cast<uint32_t *>(stg_ptr + 2048 + (2 * j + (lane & 1)) * 64 +
                                                          (((lane >> 3) ^ (j & 3)) << 4) + ((lane >> 1) & 3) * 4) =
                                lane & 1 ? __byte_perm(other, h[j], 0x7632) : __byte_perm(h[j], other, 0x5410);
                        }
                    }
                    ptx::fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        ptx::tma_store_2d(map, stg, col0, row0);
                        if (t.mirror) ptx::tma_store_2d(map, stg + 2048, row0, col0);
                        ptx::bulk_commit_group();
                    }
                    if (!more) return;
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[j]));
                        v[2 * j] -= f.x, v[2 * j + 1] -= f.y;
                    }
                };
                store(&g.map[t.prob][4], lows);
                if (lows) store(&g.map[t.prob][5], false);
            }
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) cluster::mbar_arrive(b ? leader_tempty1 : leader_tempty0);
        }
        if (lane == 0) ptx::bulk_wait_all();  // stores done before the staging buffer goes away
    }

    ptx::tc_fence_before();
    __syncthreads();
    cluster::sync();  // no CTA leaves while its peer may still touch its memory
    if (warp == 1) {
        ptx::tc_fence_after();
        pair::tmem_dealloc2(tmem, 512);
    }
}

}  // namespace mma
}  // namespace muon
}  // namespace noble
