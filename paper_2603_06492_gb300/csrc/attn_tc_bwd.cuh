// Backward attention over documents on the tensor cores: two kernels, so that each sum
// has one block and a fixed order, without atomics; only dk and dv of few key heads go through
// fp32 parts in memory, which are added up in order.  Both form the scores again (seven products of the size of one score block's, where sharing them
// would take five).
//
// dq_kernel, 128 queries of a head over the key tiles that they see:
//     S = Q K^T, dP = dO V^T;  dS = P (dP - delta);  dQ += dS K
// dkv_kernel, 128 keys of a key head over the query tiles that see them, of every query
// head that shares it, or of one of `splits` parts of them, which join_kernel then adds up
// (rows of the score block are keys):
//     S = K Q^T, dP = V dO^T;  dV += P dO,  dK += dS Q
// P and dS are written as bf16 over S and dP in TMEM and read from there as operands.
// Two warpgroups of 128 rows take half of the columns each.
//
// The tensor pipe is never behind one chain of dependent steps.  dq: the next S goes to a
// second buffer, and the next dP runs as soon as this one is in registers.  dkv:
// dV and the next S run while dS is formed, dK and the next dP while the next P is.
//
// What bounds it: the warps' instructions between the products, then the tensor pipe
// (16384 tokens, 16 heads of 128, causal: dq 1.10 ms, dk and dv 1.35, 1170 TFLOP/s of five
// products; heads of 64: 0.73 and 1.02).  Short documents pay per piece as in the forward: 8 of
// 1024 tokens, 16 heads of 64: 50 and 63 us; 64 of 197, 12 heads: 53 and 68.
#pragma once

#include "attn_tc.cuh"

namespace noble {
namespace attn {
namespace tc {

struct BwdArgs {
    RowArgs<__nv_bfloat16> a;
    float *delta;  // [n_q][T]: sum of o do
    int tiles;     // of 128 tokens
    // dkv_kernel: parts that a key head's query heads are split into, of how many of them each,
    // in all; with several their fp32 results go to part, [tile][key head][split][dv, dk]
    // [features / 4][128 tokens][4]
    int splits, heads, parts;
    float *part;
    uint32_t *status;
};

// Shared memory: two resident tiles, a ring of X stages of the tensor that is used twice
// (K in dq_kernel, Q in dkv_kernel) and of Y of the other, document starts, vectors.
template <int DP, int X, int Y, uint32_t VEC, int DOCS>
struct Bwd {
    static constexpr int kThreads = 384, kXStages = X, kYStages = Y, kDocsKept = DOCS;
    static constexpr uint32_t kTile = kChunk * (DP / 64);
    static constexpr uint32_t kR0 = 0, kR1 = kTile, kX = 2 * kTile, kY = kX + X * kTile;
    static constexpr uint32_t kDocs = kY + Y * kTile;
    static constexpr uint32_t kVec = kDocs + 2 * DOCS * 4;
    static constexpr uint32_t kBars = kVec + VEC;
    static constexpr int kNumBars = 3 * X + 5 * Y + 12;
    static constexpr uint32_t kWork = kBars + 8 * ((kNumBars + 1) & ~1);
    static constexpr uint32_t kAgain = kWork + Work::kBytes + 16;
    static constexpr uint32_t kBytes = kAgain + Again::kBytes;
    static_assert(kBytes <= 232448, "shared memory of a block");
};
// A K tile is in use from its S to its dQ, a step and a half: with 128 features a third
// stage leaves its load the time it takes (3327 clocks a tile with two, of which 1080
// waiting for it).
template <int DP> using BwdQ = Bwd<DP, DP == 64 ? 4 : 3, DP == 64 ? 4 : 2, 1024, 128>;
constexpr uint32_t kVecBytes = 128 * 8;  // lse, delta [128]
template <int DP> using BwdKV = Bwd<DP, DP == 64 ? 4 : 2, DP == 64 ? 4 : 2, (DP == 64 ? 4 : 2) * kVecBytes, kDocsInSmem>;

// Queries that see any key of [j0, j1): none if lo >= hi.
__device__ __forceinline__ Range queries_of(const Mask &m, int j0, int j1)
{
    const int end = docs_end(m);
    j1 = min(j1, end);
    if (j0 >= j1) return {0, 0};
    auto doc = [&](int j) {  // its document, as one start after another
        int a = -1, b = m.n_docs + 1;
        while (b - a > 1) {
            const int c = (a + b) >> 1;
            if (m.doc_start[c] <= j) a = c;
            else b = c;
        }
        return a;
    };
    Range r;
    const int a = doc(j0);
    if (a < 0) {
        r.lo = clampi(m.doc_start[0], 0, m.T);
    } else {
        const int s = clampi(m.doc_start[a], 0, m.T), e = clampi(m.doc_start[a + 1], s, m.T);
        if (!m.causal) r.lo = m.window ? max(s, j0 - m.window + 1) : s;
        else r.lo = m.prefix && j0 < s + clampi(m.prefix[a], 0, e - s) ? s : j0;
    }
    const int z = doc(j1 - 1);
    if (z < 0) return {0, 0};
    const int s = clampi(m.doc_start[z], 0, m.T), e = clampi(m.doc_start[z + 1], s, m.T);
    r.hi = m.window ? min(e, j1 - 1 + m.window) : e;
    return r;
}

// Those that see key j.
__device__ __forceinline__ Range queries_of(const Mask &m, int j)
{
    if (j >= docs_end(m)) return {0, 0};
    int a = -1, b = m.n_docs + 1;
    while (b - a > 1) {
        const int c = (a + b) >> 1;
        if (m.doc_start[c] <= j) a = c;
        else b = c;
    }
    if (a < 0) return {0, 0};
    const int s = clampi(m.doc_start[a], 0, m.T), e = clampi(m.doc_start[a + 1], s, m.T);
    Range r = {s, m.window ? min(e, j + m.window) : e};
    if (!m.causal) r.lo = m.window ? max(s, j - m.window + 1) : s;
    else if (!m.prefix || j >= s + clampi(m.prefix[a], 0, e - s)) r.lo = j;
    return r;
}

// ---------------------------------------------------------------- dq
template <int DP, bool GENERAL>
__global__ void __launch_bounds__(384, 1)
dq_kernel(const __grid_constant__ CUtensorMap mQ, const __grid_constant__ CUtensorMap mDO, const __grid_constant__ CUtensorMap mK,
          const __grid_constant__ CUtensorMap mV, const __grid_constant__ BwdArgs args)
{
    using B = BwdQ<DP>;
    constexpr int kXS = B::kXStages, kYS = B::kYStages, kChunks = DP / 64;
    constexpr uint32_t kS0 = 0, kDP = 128, kS1 = 256, kAcc = 384;  // TMEM columns
    extern __shared__ __align__(1024) uint8_t smem[];  // nothing static: begins on the 1024 bytes of a swizzled tile
    const uint32_t base = ptx::smem_u32(smem);
    if (base & 1023u) {
        if (threadIdx.x == 0) raise_status(args.status, kStatusBadShape);
        return;
    }
    const uint32_t bars = base + B::kBars;
    auto k_full = [&](int s) { return bars + 8u * s; };
    auto k_empty = [&](int s) { return bars + 8u * (kXS + s); };
    auto v_full = [&](int s) { return bars + 8u * (2 * kXS + s); };
    auto v_empty = [&](int s) { return bars + 8u * (2 * kXS + kYS + s); };
    const uint32_t one = bars + 8u * (2 * kXS + 2 * kYS);
    const uint32_t q_full = one, q_empty = one + 8, dp_full = one + 16, dp_read = one + 24, acc_full = one + 32,
                   acc_empty = one + 40, sums = one + 48;
    // By S buffer, since both run a step ahead: the next S does not wait for this one's
    // readers, and a warp can be through with the next dS while another is at this one.
    auto s_full = [&](int i) { return one + 56 + 8u * (i & 1); };
    auto ds_full = [&](int i) { return one + 72 + 8u * (i & 1); };
    Padding pad_k{one + 88, 0}, pad_v{pad_k.at(kXS), 0};
    const Work works{base + B::kWork};
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + B::kWork + Work::kBytes);
    const Again again{reinterpret_cast<uint32_t *>(smem + B::kAgain)};
    float *part = reinterpret_cast<float *>(smem + B::kVec);  // [2][128]
    const int warp = (int)uniform(threadIdx.x / 32), lane = threadIdx.x % 32;
    uint32_t *status = args.status;

    if (warp == 8 && lane == 0) {
        ptx::tma_prefetch_desc(&mQ);
        ptx::tma_prefetch_desc(&mDO);
        ptx::tma_prefetch_desc(&mK);
        ptx::tma_prefetch_desc(&mV);
        for (int s = 0; s < kXS; ++s) {
            ptx::mbar_init(k_full(s), 1);
            ptx::mbar_init(k_empty(s), 1);
            ptx::mbar_init(pad_k.at(s), 1);
        }
        for (int s = 0; s < kYS; ++s) {
            ptx::mbar_init(v_full(s), 1);
            ptx::mbar_init(v_empty(s), 1);
            ptx::mbar_init(pad_v.at(s), 1);
        }
        ptx::mbar_init(q_full, 1);
        ptx::mbar_init(q_empty, 1);
        ptx::mbar_init(s_full(0), 1);
        ptx::mbar_init(s_full(1), 1);
        ptx::mbar_init(dp_full, 1);
        ptx::mbar_init(dp_read, 8);
        ptx::mbar_init(ds_full(0), 8);
        ptx::mbar_init(ds_full(1), 8);
        ptx::mbar_init(acc_full, 1);
        ptx::mbar_init(acc_empty, 8);
        ptx::mbar_init(sums, 8);
        works.init(11);
        ptx::fence_barrier_init();
    }
    if (warp == 9) {
        ptx::tmem_alloc(ptx::smem_u32(tmem_slot), 512);
        ptx::tmem_relinquish();
    }
    again.init();
    const Mask mask = mask_in_smem<B::kDocsKept>(args.a.mask, reinterpret_cast<int32_t *>(smem + B::kDocs));
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = uniform(*tmem_slot);

    // piece of work: 128 queries from i0 of head h over keys from lo, `steps` tiles
    struct Rows {
        int i0, h, g, lo, steps;
    };
    auto as_rows = [](const Piece &p) { return Rows{p.v[0], p.v[1], p.v[2], p.v[3], p.v[4]}; };
    auto describe = [&](int work) {
        const int h = work % args.a.n_q, i0 = (args.tiles - 1 - work / args.a.n_q) * kRows;
        const int lo = visible(mask, i0).lo, hi = visible(mask, min(i0 + kRows, mask.T) - 1).hi;
        return Piece{{i0, h, h / (args.a.n_q / args.a.n_kv), lo, (max(hi - lo, 0) + kRows - 1) / kRows, 0, 0, 0}};
    };
    Piece pc;

    if (warp >= 8) {
        setmaxnreg_dec<88>();
        const int padding = padding_from(mask);
        auto padded = [&](const Rows &p) { return p.lo + p.steps * kRows > padding; };  // its last tile
        if (warp == 8 && lane == 0) {
            // ---------------- loads
            int n = 0, items = 0, nk = 0;
            bool ok = true;
            for (int w = 0; ok && works.take(pc, w, false, true, 0, status); ++w) {
                const Rows p = as_rows(pc);
                if (!p.steps) continue;
                ok = ptx::mbar_wait(q_empty, (items & 1) ^ 1, status);
                if (!ok) break;
                ptx::mbar_arrive_expect_tx(q_full, 2 * B::kTile);
                for (int c = 0; c < kChunks; ++c) {
                    tma_load_3d(base + B::kR0 + c * kChunk, &mQ, q_full, 64 * c, p.h, p.i0);
                    tma_load_3d(base + B::kR1 + c * kChunk, &mDO, q_full, 64 * c, p.h, p.i0);
                }
                ++items;
                for (int t = 0; t < p.steps; ++t, ++n) {
                    const int sx = n % kXS, sy = n % kYS, j = p.lo + t * kRows;
                    ok = ptx::mbar_wait(k_empty(sx), ((n / kXS) & 1) ^ 1, status);
                    if (!ok) break;
                    const bool pad = t + 1 == p.steps && padded(p);
                    const uint32_t to_k = pad ? pad_k.at(sx) : k_full(sx), to_v = pad ? pad_v.at(sy) : v_full(sy);
                    ptx::mbar_arrive_expect_tx(to_k, B::kTile);
                    for (int c = 0; c < kChunks; ++c) tma_load_3d(base + B::kX + sx * B::kTile + c * kChunk, &mK, to_k, 64 * c, p.g, j);
                    ++nk;
                    ok = ptx::mbar_wait(v_empty(sy), ((n / kYS) & 1) ^ 1, status);
                    if (!ok) break;
                    ptx::mbar_arrive_expect_tx(to_v, B::kTile);
                    for (int c = 0; c < kChunks; ++c) tma_load_3d(base + B::kY + sy * B::kTile + c * kChunk, &mV, to_v, 64 * c, p.g, j);
                }
            }
            if (items) ptx::mbar_wait(q_full, (items - 1) & 1, nullptr);
            for (int i = max(nk - kXS, 0); i < nk; ++i) ptx::mbar_wait(k_full(i % kXS), (i / kXS) & 1, nullptr);
            for (int i = max(n - kYS, 0); i < n; ++i) ptx::mbar_wait(v_full(i % kYS), (i / kYS) & 1, nullptr);
        } else if (warp == 9) {
            // ---------------- products
            const bool leader = elect_one();
            constexpr uint32_t id_s = ptx::idesc_bf16(128, 128, false, false), id_q = ptx::idesc_bf16(128, DP, false, true);
            const uint32_t dr0 = desc_k(base + B::kR0), dr1 = desc_k(base + B::kR1), dx = desc_k(base + B::kX),
                           dy = desc_k(base + B::kY), dm = desc_mn(base + B::kX);
            constexpr uint32_t kStep = B::kTile >> 4;
            // rings by index and parity: K of the next S, of the next dQ; V; steps' parities
            uint32_t st_s = 0, ph_s = 0, st_q = 0, st_v = 0, ph_v = 0, i_s = 0, i_p = 0, i_q = 0;
            int items = 0;
            auto next = [](uint32_t i, uint32_t n) { return i + 1 == n ? 0u : i + 1; };
            auto score = [&] {
                if (!wait_warp(k_full(st_s), ph_s, status)) return false;
                ptx::tc_fence_after();
                if (leader) {
                    product_features<DP>(tmem + (i_s & 1 ? kS1 : kS0), dr0, dx + st_s * kStep, id_s);
                    ptx::mma_commit(s_full(i_s));
                }
                st_s = next(st_s, kXS), ph_s ^= st_s == 0, ++i_s;
                return true;
            };
            auto dprob = [&](bool last) {  // once the dP before is in registers
                if (!wait_warp(v_full(st_v), ph_v, status) || (i_p > 0 && !wait_warp(dp_read, (i_p - 1) & 1, status))) return false;
                ptx::tc_fence_after();
                if (leader) {
                    product_features<DP>(tmem + kDP, dr1, dy + st_v * kStep, id_s);
                    ptx::mma_commit(dp_full);
                    ptx::mma_commit(v_empty(st_v));
                    if (last) ptx::mma_commit(q_empty);  // the last use of Q and dO
                }
                st_v = next(st_v, kYS), ph_v ^= st_v == 0, ++i_p;
                return true;
            };
            bool ok = true;
            for (int w = 0; ok && works.take(pc, w, true, false, lane, status); ++w) {
                const Rows p = as_rows(pc);
                if (!p.steps) continue;
                ok = wait_warp(q_full, items & 1, status) && score() && dprob(p.steps == 1);
                for (int t = 0; ok && t < p.steps; ++t) {
                    // S over the dS that the product before last has read
                    if (t + 1 < p.steps) ok = score() && dprob(t + 2 == p.steps);
                    ok = ok && wait_warp(ds_full(i_q), (i_q >> 1) & 1, status) && (t > 0 || wait_warp(acc_empty, (items & 1) ^ 1, status));
                    if (!ok) break;
                    ptx::tc_fence_after();
                    const uint32_t ds = tmem + (i_q & 1 ? kS1 : kS0);
                    if (leader) {
                        product_tokens(tmem + kAcc, ds, ds + 64, dm + st_q * kStep, id_q, t > 0);
                        ptx::mma_commit(k_empty(st_q));
                    }
                    st_q = next(st_q, kXS), ++i_q;
                }
                if (leader) ptx::mma_commit(acc_full);
                ++items;
            }
            // every product has finished before TMEM is released below
            if (items) ptx::mbar_wait(acc_full, (items - 1) & 1, nullptr);
        } else if (warp == 10 && lane == 0) {
            works.hand_out(describe, again.any(), status);
        } else if (warp == 11) {
            // ---------------- padding
            int n = 0;
            for (int w = 0; works.take(pc, w, true, false, lane, status); ++w) {
                const Rows p = as_rows(pc);
                n += p.steps;
                if (p.steps == 0 || !padded(p)) continue;
                const int sx = (n - 1) % kXS, sy = (n - 1) % kYS, from = padding - (p.lo + (p.steps - 1) * kRows);
                if (!pad_k.clear<DP>(smem + B::kX + sx * B::kTile, sx, from, k_full(sx), lane, status)) break;
                if (!pad_v.clear<DP>(smem + B::kY + sy * B::kTile, sy, from, v_full(sy), lane, status)) break;
            }
        }
        __syncwarp();
    } else {
        // ---------------- dS: thread = row and half of the columns
        setmaxnreg_inc<208>();
        const int half = warp / 4, row = threadIdx.x % 128;
        const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
        const float sl = args.a.score.scale * kLog2e;
        uint32_t n = 0, items = 0, nsums = 0;
        bool ok = true;
        // a piece's row: its values are on their way while the piece before is written out
        struct Row {
            Rows p;
            Range rg;
            float lse, delta;
        } r;
        auto fetch = [&](Row &r) {
            r.p = as_rows(pc);
            const int i = r.p.i0 + row;
            const bool real = i < mask.T;
            const int64_t at = (int64_t)r.p.h * mask.T + i;
            r.lse = real ? args.a.lse[at] : 0.f;
            r.delta = real ? args.delta[at] : 0.f;
            r.rg = real ? visible(mask, i) : Range{0, 0};
        };
        bool more = works.take(pc, 0, true, false, lane, status);
        if (more) fetch(r);
        for (int w = 1; ok && more; ++w) {
            const Rows p = r.p;
            const Range rg = r.rg;
            const int i = p.i0 + row;
            const bool real = i < mask.T, none = rg.lo >= rg.hi;
            const int64_t at = (int64_t)p.h * mask.T + (real ? i : 0);
            const float lse2 = none ? 0.f : r.lse * kLog2e;
            float delta = none ? 0.f : r.delta;
            const float slope = GENERAL && args.a.score.slope ? args.a.score.slope[p.h] * kLog2e : 0.f;
            for (int t = 0; t < p.steps; ++t, ++n) {
                const uint32_t tS = tmem + lanes + (n & 1 ? kS1 : kS0) + 64 * half, tP = tmem + lanes + kDP + 64 * half;
                const int j0 = p.lo + t * kRows + 64 * half;
                ok = ptx::mbar_wait(s_full(n), (n >> 1) & 1, status) && ptx::mbar_wait(dp_full, n & 1, status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                ptx::tc_fence_after();
                uint32_t xs[64], xp[64];
                __syncwarp();
                tmem_ld32(tS, xs);
                tmem_ld32(tS + 32, xs + 32);
                tmem_ld32(tP, xp);
                tmem_ld32(tP + 32, xp + 32);
                tmem_wait_ld();
                pin32(xs), pin32(xs + 32), pin32(xp), pin32(xp + 32);
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(dp_read);
                float s[64], dp[64];
                as_floats(s, xs);
                as_floats(dp, xp);
                uint32_t pk[32];
                const int lo = rg.lo - j0, hi = rg.hi - j0;
                const bool all = __all_sync(0xffffffffu, lo <= 0 && hi >= 64);
                auto total = [&](float sum) {  // over both threads of a row; in a bounded wait's time
                    part[128 * half + row] = sum;
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(sums);
                    ok = ptx::mbar_wait(sums, nsums & 1, status);
                    ok = __all_sync(0xffffffffu, ok);
                    ++nsums;
                    return part[row] + part[128 + row];
                };
                // With one step, all that the row sees is here: delta is then summed from p and dp
                // themselves (see simt::dq_kernel).
                if (!GENERAL) {
                    // p over s, and 0 where nothing is seen
                    const uint64_t sl2 = pack2(sl, sl), l2 = pack2(-lse2, -lse2);
#pragma unroll
                    for (int c = 0; c < 64; c += 2) {
                        float a, b;
                        unpack2(fma2(pack2(s[c], s[c + 1]), sl2, l2), a, b);
                        s[c] = exp2_fast(a), s[c + 1] = exp2_fast(b);
                    }
                    if (!all)
#pragma unroll
                        for (int c = 0; c < 64; ++c) {
                            const bool in = c >= lo && c < hi;
                            s[c] = in ? s[c] : 0.f;  // dp is finite, or the row is done again
                        }
                    if (p.steps == 1) {
                        float sum = 0.f;
#pragma unroll
                        for (int c = 0; c < 64; ++c) sum = fmaf(s[c], c >= lo && c < hi ? dp[c] : 0.f, sum);
                        delta = total(sum);
                    }
                    const uint64_t d2 = pack2(-delta, -delta);
#pragma unroll
                    for (int c = 0; c < 64; c += 2) {
                        float a, b;
                        unpack2(mul2(pack2(s[c], s[c + 1]), add2(pack2(dp[c], dp[c + 1]), d2)), a, b);
                        pk[c / 2] = ptx::pack_bf16x2(a, b);
                    }
                } else {
                    // a pair of columns at a time from score to dS, since the derivatives have no room beside both
                    const Capping cap = capping(s, args.a.score, !none);
                    const float far = (float)(i - j0);
                    const uint64_t far2 = pack2(far, far), l2 = pack2(-lse2, -lse2), slope2 = pack2(-slope, -slope);
                    auto as_ds = [&](auto mode, auto biased) {
                        auto probs = [&](int c, uint64_t &x, uint64_t &g) {
                            x = pack2(s[c], s[c + 1]);
                            cap_pair<mode.value, true>(x, g, cap);
                            if constexpr (decltype(biased)::value) {
                                const uint64_t by = add2(far2, pack2(-(float)c, -(float)(c + 1))) & 0x7fffffff7fffffffull;
                                x = fma2(slope2, by, x);
                            }
                            float a, b;
                            unpack2(add2(x, l2), a, b);
                            x = pack2(exp2_fast(a), exp2_fast(b));
                        };
                        if (p.steps == 1) {
                            float sum = 0.f;
#pragma unroll
                            for (int c = 0; c < 64; c += 2) {
                                uint64_t v, g;
                                float x, y;
                                probs(c, v, g);
                                unpack2(v, x, y);
                                sum += c >= lo && c < hi ? x * dp[c] : 0.f;
                                sum += c + 1 >= lo && c + 1 < hi ? y * dp[c + 1] : 0.f;
                            }
                            delta = total(sum);
                        }
                        const uint64_t d2 = pack2(-delta, -delta);
#pragma unroll
                        for (int c = 0; c < 64; c += 2) {
                            uint64_t v, g;
                            float x, y;
                            probs(c, v, g);
                            unpack2(mul2(mul2(v, g), add2(pack2(dp[c], dp[c + 1]), d2)), x, y);
                            if (!all) x = c >= lo && c < hi ? x : 0.f, y = c + 1 >= lo && c + 1 < hi ? y : 0.f;
                            pk[c / 2] = ptx::pack_bf16x2(x, y);
                        }
                    };
                    with_cap(cap.mode, [&](auto mode) {
                        if (args.a.score.slope) as_ds(mode, std::true_type{});
                        else as_ds(mode, std::false_type{});
                    });
                }
                if (!ok) break;
                if (p.steps == 1 && half == 0 && !none) args.delta[at] = delta;
                __syncwarp();
                tmem_st32(tS, pk);
                tmem_wait_st();
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(ds_full(n));
            }
            if (!ok) break;
            more = works.take(pc, w, true, false, lane, status);
            if (more) fetch(r);
            // ---------------- dq of this row, half of its features
            if (p.steps) {
                ok = ptx::mbar_wait(acc_full, items & 1, status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                ++items;
                ptx::tc_fence_after();
            }
            bool fine = true;
            __nv_bfloat16 *out = args.a.dq.at(i - lane, p.h) + half * (DP / 2);
#pragma unroll 1
            for (int c = 0; c < DP / 2; c += 32) {
                uint32_t o[32];
                if (p.steps) {
                    __syncwarp();
                    tmem_ld32(tmem + lanes + kAcc + half * (DP / 2) + c, o);
                    tmem_wait_ld();
                    pin32(o);
                    ptx::tc_fence_before();
                    __syncwarp();
                    if (lane == 0 && c + 32 == DP / 2) ptx::mbar_arrive(acc_empty);
                }
                fine &= write_rows(o, args.a.score.scale, none || !p.steps, out + c, args.a.dq.row, mask.T - (i - lane),
                                   args.a.d - half * (DP / 2) - c, lane);
            }
            again.note(warp, lane, i - lane, p.h, __ballot_sync(0xffffffffu, real && !fine));
        }
        // half of a row's features, as the warp that noted it; delta in memory is this kernel's by now
        again.each(warp, [&](int w, int i, int h) {
            const int f = w / 4 * (DP / 2);
            row_dq(args.a, i, h, lane, args.delta[(int64_t)h * mask.T + i], f, f + DP / 2);
        });
    }

    ptx::tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, 512);
    }
}

// ---------------------------------------------------------------- dk, dv
template <int DP, bool GENERAL>
__global__ void __launch_bounds__(384, 1)
dkv_kernel(const __grid_constant__ CUtensorMap mQ, const __grid_constant__ CUtensorMap mDO, const __grid_constant__ CUtensorMap mK,
           const __grid_constant__ CUtensorMap mV, const __grid_constant__ BwdArgs args)
{
    using B = BwdKV<DP>;
    constexpr int kStages = B::kXStages, kChunks = DP / 64;
    constexpr uint32_t kS = 0, kDP = 128, kDV = 256, kDK = 256 + DP;  // TMEM columns
    extern __shared__ __align__(1024) uint8_t smem[];  // as in dq_kernel
    const uint32_t base = ptx::smem_u32(smem);
    if (base & 1023u) {
        if (threadIdx.x == 0) raise_status(args.status, kStatusBadShape);
        return;
    }
    const uint32_t bars = base + B::kBars;
    auto q_full = [&](int s) { return bars + 8u * s; };
    auto q_empty = [&](int s) { return bars + 8u * (kStages + s); };
    auto o_full = [&](int s) { return bars + 8u * (2 * kStages + s); };
    auto o_empty = [&](int s) { return bars + 8u * (3 * kStages + s); };
    auto vec_full = [&](int s) { return bars + 8u * (4 * kStages + s); };
    auto vec_empty = [&](int s) { return bars + 8u * (5 * kStages + s); };
    const uint32_t one = bars + 8u * (6 * kStages);
    const uint32_t kv_full = one, kv_empty = one + 8, s_full = one + 16, dp_full = one + 24, p_full = one + 32, ds_full = one + 40,
                   acc_full = one + 48, acc_empty = one + 56;
    Padding pad_q{one + 64, 0}, pad_o{pad_q.at(kStages), 0};
    const Work works{base + B::kWork};
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + B::kWork + Work::kBytes);
    const Again again{reinterpret_cast<uint32_t *>(smem + B::kAgain)};
    const int warp = (int)uniform(threadIdx.x / 32), lane = threadIdx.x % 32;
    uint32_t *status = args.status;

    if (warp == 8 && lane == 0) {
        ptx::tma_prefetch_desc(&mQ);
        ptx::tma_prefetch_desc(&mDO);
        ptx::tma_prefetch_desc(&mK);
        ptx::tma_prefetch_desc(&mV);
        for (int s = 0; s < kStages; ++s) {
            ptx::mbar_init(q_full(s), 1);
            ptx::mbar_init(q_empty(s), 1);
            ptx::mbar_init(o_full(s), 1);
            ptx::mbar_init(o_empty(s), 1);
            ptx::mbar_init(vec_full(s), 1);
            ptx::mbar_init(vec_empty(s), 8);
            ptx::mbar_init(pad_q.at(s), 1);
            ptx::mbar_init(pad_o.at(s), 1);
        }
        ptx::mbar_init(kv_full, 1);
        ptx::mbar_init(kv_empty, 1);
        ptx::mbar_init(s_full, 1);
        ptx::mbar_init(dp_full, 1);
        ptx::mbar_init(p_full, 8);
        ptx::mbar_init(ds_full, 8);
        ptx::mbar_init(acc_full, 1);
        ptx::mbar_init(acc_empty, 8);
        works.init(11);
        ptx::fence_barrier_init();
    }
    if (warp == 9) {
        ptx::tmem_alloc(ptx::smem_u32(tmem_slot), 512);
        ptx::tmem_relinquish();
    }
    again.init();
    const Mask mask = mask_in_smem<B::kDocsKept>(args.a.mask, reinterpret_cast<int32_t *>(smem + B::kDocs));
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = uniform(*tmem_slot);

    // piece of work: 128 keys from j0 of key head g, over query tiles from lo, `per` of a
    // head and `steps` in all, of the query heads from h0
    struct Keys {
        int j0, g, lo, per, steps, h0, part;
    };
    auto as_keys = [](const Piece &p) { return Keys{p.v[0], p.v[1], p.v[2], p.v[3], p.v[4], p.v[5], p.v[6]}; };
    auto describe = [&](int work) {
        const int tile = work / args.parts, part = work - tile * args.parts, j0 = tile * kRows;
        const Range r = queries_of(mask, j0, j0 + kRows);
        const int per = (max(r.hi - r.lo, 0) + kRows - 1) / kRows;
        return Piece{{j0, args.splits == 1 ? part : part / args.splits, r.lo, per, per * args.heads, part * args.heads, part, 0}};
    };
    Piece pc;

    if (warp >= 8) {
        setmaxnreg_dec<88>();
        const int padding = padding_from(mask);
        // the last tile of every head
        auto padded = [&](const Keys &p, int t) { return p.lo + p.per * kRows > padding && (t + 1) % p.per == 0; };
        if (warp == 8 && lane == 0) {
            // ---------------- loads
            int n = 0, items = 0, nq = 0;
            bool ok = true;
            for (int w = 0; ok && works.take(pc, w, false, true, 0, status); ++w) {
                const Keys p = as_keys(pc);
                if (!p.steps) continue;
                ok = ptx::mbar_wait(kv_empty, (items & 1) ^ 1, status);
                if (!ok) break;
                ptx::mbar_arrive_expect_tx(kv_full, 2 * B::kTile);
                for (int c = 0; c < kChunks; ++c) {
                    tma_load_3d(base + B::kR0 + c * kChunk, &mK, kv_full, 64 * c, p.g, p.j0);
                    tma_load_3d(base + B::kR1 + c * kChunk, &mV, kv_full, 64 * c, p.g, p.j0);
                }
                ++items;
                for (int t = 0; t < p.steps; ++t, ++n) {
                    const int st = n % kStages, h = p.h0 + t / p.per, i = p.lo + t % p.per * kRows;
                    const uint32_t ph = (n / kStages) & 1;
                    ok = ptx::mbar_wait(q_empty(st), ph ^ 1, status);
                    if (!ok) break;
                    const bool pad = padded(p, t);
                    const uint32_t to_q = pad ? pad_q.at(st) : q_full(st), to_o = pad ? pad_o.at(st) : o_full(st);
                    ptx::mbar_arrive_expect_tx(to_q, B::kTile);
                    for (int c = 0; c < kChunks; ++c) tma_load_3d(base + B::kX + st * B::kTile + c * kChunk, &mQ, to_q, 64 * c, h, i);
                    ++nq;
                    ok = ptx::mbar_wait(o_empty(st), ph ^ 1, status);
                    if (!ok) break;
                    ptx::mbar_arrive_expect_tx(to_o, B::kTile);
                    for (int c = 0; c < kChunks; ++c) tma_load_3d(base + B::kY + st * B::kTile + c * kChunk, &mDO, to_o, 64 * c, h, i);
                }
            }
            if (items) ptx::mbar_wait(kv_full, (items - 1) & 1, nullptr);
            for (int i = max(nq - kStages, 0); i < nq; ++i) ptx::mbar_wait(q_full(i % kStages), (i / kStages) & 1, nullptr);
            for (int i = max(n - kStages, 0); i < n; ++i) ptx::mbar_wait(o_full(i % kStages), (i / kStages) & 1, nullptr);
        } else if (warp == 9) {
            // ---------------- products
            const bool leader = elect_one();
            constexpr uint32_t id_s = ptx::idesc_bf16(128, 128, false, false), id_d = ptx::idesc_bf16(128, DP, false, true);
            int n = 0, items = 0;
            bool ok = true;
            for (int w = 0; ok && works.take(pc, w, true, false, lane, status); ++w) {
                const Keys p = as_keys(pc);
                if (!p.steps) continue;
                const uint32_t dr0 = desc_k(base + B::kR0), dr1 = desc_k(base + B::kR1), dx = desc_k(base + B::kX),
                               dy = desc_k(base + B::kY), mx = desc_mn(base + B::kX), my = desc_mn(base + B::kY);
                constexpr uint32_t kStep = B::kTile >> 4;
                auto score = [&](int i) {
                    if (!wait_warp(q_full(i % kStages), (i / kStages) & 1, status)) return false;
                    ptx::tc_fence_after();
                    if (leader) product_features<DP>(tmem + kS, dr0, dx + (i % kStages) * kStep, id_s);
                    if (leader) ptx::mma_commit(s_full);
                    return true;
                };
                auto dprob = [&](int i) {
                    if (!wait_warp(o_full(i % kStages), (i / kStages) & 1, status)) return false;
                    ptx::tc_fence_after();
                    if (leader) product_features<DP>(tmem + kDP, dr1, dy + (i % kStages) * kStep, id_s);
                    if (leader) ptx::mma_commit(dp_full);
                    if (i == n + p.steps - 1 && leader) ptx::mma_commit(kv_empty);  // the last use of K and V
                    return true;
                };
                ok = wait_warp(kv_full, items & 1, status) && score(n) && dprob(n);
                for (int t = 0; ok && t < p.steps; ++t) {
                    const int i = n + t;
                    ok = wait_warp(p_full, i & 1, status) && (t > 0 || wait_warp(acc_empty, (items & 1) ^ 1, status));
                    if (!ok) break;
                    ptx::tc_fence_after();
                    if (leader) product_tokens(tmem + kDV, tmem + kS, tmem + kS + 64, my + (i % kStages) * kStep, id_d, t > 0);
                    if (leader) ptx::mma_commit(o_empty(i % kStages));
                    if (t + 1 < p.steps) ok = score(i + 1);  // over P, read by then: products run in order
                    ok = ok && wait_warp(ds_full, i & 1, status);
                    if (!ok) break;
                    ptx::tc_fence_after();
                    if (leader) product_tokens(tmem + kDK, tmem + kDP, tmem + kDP + 64, mx + (i % kStages) * kStep, id_d, t > 0);
                    if (leader) ptx::mma_commit(q_empty(i % kStages));
                    if (t + 1 < p.steps) ok = dprob(i + 1);  // over dS
                }
                if (!ok) break;
                if (leader) ptx::mma_commit(acc_full);
                n += p.steps;
                ++items;
            }
            // every product has finished before TMEM is released below
            if (items) wait_warp(acc_full, (items - 1) & 1, nullptr);
        } else if (warp == 10) {
            // ---------------- lse and delta of the query tiles, a step ahead of the stage they go to;
            // their padding
            int n = 0;
            bool ok = true;
            const int end = docs_end(mask);
            for (int w = 0; ok && works.take(pc, w, true, false, lane, status); ++w) {
                const Keys p = as_keys(pc);
                float lse[4], delta[4];
                auto fetch = [&](int t) {
                    const int h = p.h0 + t / p.per, i0 = p.lo + t % p.per * kRows;
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int i = i0 + lane + 32 * u;
                        const int64_t at = (int64_t)h * mask.T + i;
                        lse[u] = i < end ? args.a.lse[at] : 0.f;
                        delta[u] = i < end ? args.delta[at] : 0.f;
                    }
                };
                if (p.steps) fetch(0);
                for (int t = 0; t < p.steps; ++t, ++n) {
                    const int st = n % kStages;
                    ok = wait_warp(vec_empty(st), ((n / kStages) & 1) ^ 1, status);
                    if (ok && padded(p, t)) {
                        const int from = padding - (p.lo + (p.per - 1) * kRows);
                        ok = pad_q.clear<DP>(smem + B::kX + st * B::kTile, st, from, q_full(st), lane, status) &&
                             pad_o.clear<DP>(smem + B::kY + st * B::kTile, st, from, o_full(st), lane, status);
                    }
                    if (!ok) break;
                    float *vec = reinterpret_cast<float *>(smem + B::kVec + st * kVecBytes);
#pragma unroll
                    for (int u = 0; u < 4; ++u) vec[lane + 32 * u] = lse[u] * kLog2e, vec[128 + lane + 32 * u] = delta[u];
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(vec_full(st));
                    if (t + 1 < p.steps) fetch(t + 1);
                }
            }
        } else if (warp == 11 && lane == 0) {
            works.hand_out(describe, again.any(), status);
        }
        __syncwarp();
    } else {
        // ---------------- P and dS: thread = key and half of the queries
        setmaxnreg_inc<208>();
        const int half = warp / 4, row = threadIdx.x % 128;
        const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
        const uint32_t tS = tmem + lanes + kS + 64 * half, tP = tmem + lanes + kDP + 64 * half;
        const float sl = args.a.score.scale * kLog2e;
        uint32_t n = 0, items = 0;
        bool ok = true;
        // the queries that see a key are a range; a piece's is looked up before the one before
        // it is written out
        Keys p_next;
        Range see_next;
        auto fetch = [&] {
            p_next = as_keys(pc);
            const int j = p_next.j0 + row;
            see_next = queries_of(mask, j);
        };
        bool more = works.take(pc, 0, true, false, lane, status);
        if (more) fetch();
        for (int w = 1; ok && more; ++w) {
            const Keys p = p_next;
            const Range see = see_next;
            const int j = p.j0 + row;
            for (int t = 0; t < p.steps; ++t, ++n) {
                const int st = n % kStages;
                const float *vec = reinterpret_cast<const float *>(smem + B::kVec + st * kVecBytes) + 64 * half;
                const int i0 = p.lo + t % p.per * kRows + 64 * half, lo = see.lo - i0, hi = see.hi - i0;
                ok = ptx::mbar_wait(vec_full(st), (n / kStages) & 1, status) && ptx::mbar_wait(s_full, n & 1, status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                ptx::tc_fence_after();
                const bool all = __all_sync(0xffffffffu, lo <= 0 && hi >= 64);
                uint32_t xs[64], xp[64];
                __syncwarp();
                tmem_ld32(tS, xs);
                tmem_ld32(tS + 32, xs + 32);
                tmem_wait_ld();
                pin32(xs), pin32(xs + 32);
                float s[64], dp[64];
                as_floats(s, xs);
                // p over s; with a capped score, dp is to be multiplied by p and g
                uint32_t gs[GENERAL ? 32 : 1];
                if (!GENERAL) {
                    const uint64_t sl2 = pack2(sl, sl);
#pragma unroll
                    for (int c = 0; c < 64; c += 4) {
                        const float4 l = *reinterpret_cast<const float4 *>(vec + c);
                        float a, b;
                        unpack2(fma2(pack2(s[c], s[c + 1]), sl2, pack2(-l.x, -l.y)), a, b);
                        s[c] = exp2_fast(a), s[c + 1] = exp2_fast(b);
                        unpack2(fma2(pack2(s[c + 2], s[c + 3]), sl2, pack2(-l.z, -l.w)), a, b);
                        s[c + 2] = exp2_fast(a), s[c + 3] = exp2_fast(b);
                    }
                } else {
                    const int h = p.h0 + t / p.per;
                    const float slope = args.a.score.slope ? args.a.score.slope[h] * kLog2e : 0.f;
                    general_scores<64, GENERAL>(s, gs, args.a.score, slope, (float)(j - i0), see.lo < see.hi);
#pragma unroll
                    for (int c = 0; c < 64; c += 4) {
                        const float4 l = *reinterpret_cast<const float4 *>(vec + c);
                        float a, b;
                        unpack2(add2(pack2(s[c], s[c + 1]), pack2(-l.x, -l.y)), a, b);
                        s[c] = exp2_fast(a), s[c + 1] = exp2_fast(b);
                        unpack2(add2(pack2(s[c + 2], s[c + 3]), pack2(-l.z, -l.w)), a, b);
                        s[c + 2] = exp2_fast(a), s[c + 3] = exp2_fast(b);
                    }
                }
                if (!all)
#pragma unroll
                    for (int c = 0; c < 64; ++c) s[c] = c >= lo && c < hi ? s[c] : 0.f;
                uint32_t pk[32];
#pragma unroll
                for (int c = 0; c < 64; c += 2) pk[c / 2] = ptx::pack_bf16x2(s[c], s[c + 1]);
                __syncwarp();
                tmem_st32(tS, pk);
                tmem_wait_st();
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(p_full);

                ok = ptx::mbar_wait(dp_full, n & 1, status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                ptx::tc_fence_after();
                __syncwarp();
                tmem_ld32(tP, xp);
                tmem_ld32(tP + 32, xp + 32);
                tmem_wait_ld();
                pin32(xp), pin32(xp + 32);
                as_floats(dp, xp);
#pragma unroll
                for (int c = 0; c < 64; c += 4) {
                    const float4 d = *reinterpret_cast<const float4 *>(vec + 128 + c);
                    float e[4];
                    unpack2(mul2(pack2(s[c], s[c + 1]), add2(pack2(dp[c], dp[c + 1]), pack2(-d.x, -d.y))), e[0], e[1]);
                    unpack2(mul2(pack2(s[c + 2], s[c + 3]), add2(pack2(dp[c + 2], dp[c + 3]), pack2(-d.z, -d.w))), e[2], e[3]);
                    if (GENERAL) {
                        const float2 g0 = __half22float2(*reinterpret_cast<const __half2 *>(&gs[c / 2]));
                        const float2 g1 = __half22float2(*reinterpret_cast<const __half2 *>(&gs[c / 2 + 1]));
                        unpack2(mul2(pack2(e[0], e[1]), pack2(g0.x, g0.y)), e[0], e[1]);
                        unpack2(mul2(pack2(e[2], e[3]), pack2(g1.x, g1.y)), e[2], e[3]);
                    }
                    pk[c / 2] = ptx::pack_bf16x2(e[0], e[1]);
                    pk[c / 2 + 1] = ptx::pack_bf16x2(e[2], e[3]);
                }
                __syncwarp();
                tmem_st32(tP, pk);
                tmem_wait_st();
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    ptx::mbar_arrive(ds_full);
                    ptx::mbar_arrive(vec_empty(st));
                }
            }
            if (!ok) break;
            more = works.take(pc, w, true, false, lane, status);
            if (more) fetch();
            // ---------------- dv by the first warpgroup, dk by the second
            if (p.steps) {
                ok = ptx::mbar_wait(acc_full, items & 1, status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                ++items;
                ptx::tc_fence_after();
            }
            const bool real = j < mask.T, none = see.lo >= see.hi;
            const float f = half ? args.a.score.scale : 1.f;
            const Heads<__nv_bfloat16> &to = half ? args.a.dk : args.a.dv;
            __nv_bfloat16 *out = to.at(j - lane, p.g);
            bool fine = true;
#pragma unroll 1
            for (int c = 0; c < DP; c += 32) {
                uint32_t o[32];
                if (p.steps) {
                    __syncwarp();
                    tmem_ld32(tmem + lanes + (half ? kDK : kDV) + c, o);
                    tmem_wait_ld();
                    pin32(o);
                    ptx::tc_fence_before();
                    __syncwarp();
                    if (lane == 0 && c + 32 == DP) ptx::mbar_arrive(acc_empty);
                }
                if (args.splits == 1) {
                    fine &= write_rows(o, f, none || !p.steps, out + c, to.row, mask.T - (j - lane), args.a.d - c, lane);
                } else {
                    const int64_t unit = (int64_t)(p.j0 / kRows) * args.parts + p.part;
                    uint4 *part = reinterpret_cast<uint4 *>(args.part) + ((unit * 2 + half) * (DP / 4) + c / 4) * kRows + row;
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        part[e / 4 * kRows] = p.steps && !none ? make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]) : make_uint4(0, 0, 0, 0);
                }
            }
            again.note(warp, lane, j - lane, p.g, __ballot_sync(0xffffffffu, real && !fine));
        }
        again.each(warp, [&](int w, int j, int g) { row_dkv(args.a, j, g, lane, w / 4 == 0, w / 4 == 1); });
    }

    ptx::tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, 512);
    }
}

// dk and dv of 128 keys from the parts of their query heads, in order: a thread per key and 32
// features.  Bound by reading the parts, most of them still in L2 (4096 tokens, 16 heads of
// 128 in four parts: 12 us).
template <int DP>
__global__ void __launch_bounds__(kRows *DP / 32) join_kernel(const __grid_constant__ BwdArgs args)
{
    __shared__ uint32_t bad[4];  // keys that are not finite, 32 a word
    const int row = threadIdx.x % kRows, chunk = threadIdx.x / kRows, warp = row / 32, lane = row % 32;
    const int half = blockIdx.x & 1, unit = blockIdx.x >> 1, g = unit % args.a.n_kv, j = unit / args.a.n_kv * kRows + row;
    if (threadIdx.x < 4) bad[threadIdx.x] = 0;
    __syncthreads();
    const Heads<__nv_bfloat16> &to = half ? args.a.dk : args.a.dv;
    const float4 *part = reinterpret_cast<const float4 *>(args.part) + (((int64_t)unit * args.splits * 2 + half) * (DP / 4) + 8 * chunk) * kRows + row;
    float4 sum[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = part[e * kRows];
    for (int s = 1; s < args.splits; ++s) {
        part += 2 * (DP / 4) * kRows;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float4 x = part[e * kRows];
            sum[e].x += x.x, sum[e].y += x.y, sum[e].z += x.z, sum[e].w += x.w;
        }
    }
    uint32_t o[32];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        o[4 * e] = __float_as_uint(sum[e].x), o[4 * e + 1] = __float_as_uint(sum[e].y), o[4 * e + 2] = __float_as_uint(sum[e].z),
              o[4 * e + 3] = __float_as_uint(sum[e].w);
    const bool fine = write_rows(o, half ? args.a.score.scale : 1.f, false, to.at(j - lane, g) + 32 * chunk, to.row,
                                 args.a.mask.T - (j - lane), args.a.d - 32 * chunk, lane);
    const uint32_t word = __ballot_sync(0xffffffffu, j < args.a.mask.T && !fine);
    if (lane == 0 && word) atomicOr(&bad[warp], word);
    __syncthreads();
    if (chunk) return;
    for (uint32_t b = bad[warp]; b; b &= b - 1) row_dkv(args.a, j - lane + __ffs(b) - 1, g, lane, half == 0, half == 1);
}

}  // namespace tc
}  // namespace attn
}  // namespace noble
