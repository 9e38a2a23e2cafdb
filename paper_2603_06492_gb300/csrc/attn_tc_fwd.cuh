// Forward attention over documents on the tensor cores.
//
// A piece of work is 256 queries of one head, as two row blocks A and B of 128, over the
// key tiles that they see:
//     S = Q K^T        operands in shared memory, S in TMEM
//     P = exp2(S - m)  one thread per row; P (bf16) over S in TMEM
//     O += P V         P from TMEM, V MN-major in shared memory
// Row blocks alternate on the tensor pipe: while one's warps compute P the pipe works on
// the other's products, and each key tile is read from L2 once for 256 queries (32 bytes
// per clock and SM at the full rate).  O stays in TMEM; it is scaled down only when a row's
// maximum has grown by more than 2^8 since the last time, which after the first tiles
// happens rarely.  Sums and maxima are fp32; P is rounded to bf16 for the product (each
// to 2^-9 of itself), its sum is that of the unrounded values.
#pragma once

#include "attn_tc.cuh"

namespace noble {
namespace attn {
namespace tc {

template <int DP>
struct Fwd {
    static constexpr int kThreads = 384;  // two softmax warpgroups; TMA, MMA, work and a spare warp
    static constexpr int kStages = DP == 64 ? 4 : 2;
    static constexpr uint32_t kTile = kChunk * (DP / 64);
    static constexpr uint32_t kQ = 0, kK = 2 * kTile, kV = kK + kStages * kTile, kDocs = kV + kStages * kTile;
    static constexpr uint32_t kBars = kDocs + 2 * kDocsInSmem * 4;
    // barriers: q full/empty, k and v full/empty by stage, s full, p full, pv done by row block, work full/empty
    static constexpr int kNumBars = 2 + 4 * kStages + 6 + 4;
    static constexpr uint32_t kWork = kBars + 8 * ((kNumBars + 1) & ~1);  // two 16-byte answers
    static constexpr uint32_t kBytes = kWork + 32 + 16;
    static constexpr uint32_t kDynamic = kBytes + 1024;
    static constexpr uint32_t kS = 0, kO = 256;  // TMEM columns: S of A and B, then O of A and B
};

struct FwdArgs {
    RowArgs<__nv_bfloat16> a;
    int tiles;  // of 256 queries
    uint32_t *status;
};

// Key tiles of a row block, counted from the first key that its piece of work sees.
struct Span {
    int i0, h, g, first, a0, a1, b0, b1;  // first key; tiles [a0, a1) of A, [b0, b1) of B
    __device__ __forceinline__ int begin() const { return a0; }
    __device__ __forceinline__ int end() const { return max(a1, b1); }
};

__device__ __forceinline__ Span fwd_span(const Mask &m, const FwdArgs &f, int work)
{
    Span s;
    s.h = work % f.a.n_q;
    s.g = s.h / (f.a.n_q / f.a.n_kv);
    s.i0 = (f.tiles - 1 - work / f.a.n_q) * 256;
    const int iA = min(s.i0 + 127, m.T - 1), iB = min(s.i0 + 255, m.T - 1);
    const Range r0 = visible(m, s.i0), rA = visible(m, iA);
    s.first = r0.lo;
    s.a0 = 0;
    s.a1 = (max(rA.hi - s.first, 0) + kRows - 1) / kRows;
    if (s.i0 + 128 < m.T) {
        const Range q0 = visible(m, s.i0 + 128), qB = visible(m, iB);
        s.b0 = (q0.lo - s.first) / kRows;
        s.b1 = (max(qB.hi - s.first, 0) + kRows - 1) / kRows;
        if (s.b1 < s.b0) s.b1 = s.b0;
    } else {
        s.b0 = s.b1 = s.a1;
    }
    return s;
}

// GENERAL: capped or biased scores, or a scale that is not positive.
template <int DP, bool GENERAL>
__global__ void __launch_bounds__(Fwd<DP>::kThreads, 1)
fwd_kernel(const __grid_constant__ CUtensorMap mQ, const __grid_constant__ CUtensorMap mK, const __grid_constant__ CUtensorMap mV,
           const __grid_constant__ FwdArgs args)
{
    using F = Fwd<DP>;
    constexpr int kStages = F::kStages, kChunks = DP / 64;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = ptx::smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (base - raw);
    const uint32_t bars = base + F::kBars;
    const uint32_t q_full = bars, q_empty = bars + 8;
    auto k_full = [&](int s) { return bars + 8u * (2 + s); };
    auto k_empty = [&](int s) { return bars + 8u * (2 + kStages + s); };
    auto v_full = [&](int s) { return bars + 8u * (2 + 2 * kStages + s); };
    auto v_empty = [&](int s) { return bars + 8u * (2 + 3 * kStages + s); };
    auto s_full = [&](int b) { return bars + 8u * (2 + 4 * kStages + b); };
    auto p_full = [&](int b) { return bars + 8u * (4 + 4 * kStages + b); };
    auto pv_done = [&](int b) { return bars + 8u * (6 + 4 * kStages + b); };
    auto w_full = [&](int s) { return bars + 8u * (8 + 4 * kStages + s); };
    auto w_empty = [&](int s) { return bars + 8u * (10 + 4 * kStages + s); };
    auto w_slot = [&](int s) { return base + F::kWork + 16u * s; };
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + F::kWork + 32);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    uint32_t *status = args.status;

    if (warp == 8 && lane == 0) {
        ptx::tma_prefetch_desc(&mQ);
        ptx::tma_prefetch_desc(&mK);
        ptx::tma_prefetch_desc(&mV);
        ptx::mbar_init(q_full, 1);
        ptx::mbar_init(q_empty, 1);
        for (int s = 0; s < kStages; ++s) {
            ptx::mbar_init(k_full(s), 1);
            ptx::mbar_init(k_empty(s), 1);
            ptx::mbar_init(v_full(s), 1);
            ptx::mbar_init(v_empty(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            ptx::mbar_init(s_full(b), 1);
            ptx::mbar_init(p_full(b), 4);
            ptx::mbar_init(pv_done(b), 1);
            ptx::mbar_init(w_full(b), 1);
            ptx::mbar_init(w_empty(b), 10);
        }
        ptx::fence_barrier_init();
    }
    if (warp == 9) {
        ptx::tmem_alloc(ptx::smem_u32(tmem_slot), 512);
        ptx::tmem_relinquish();
    }
    const Mask mask = mask_in_smem(args.a.mask, reinterpret_cast<int32_t *>(smem + F::kDocs));
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    // The next piece of work for a reader of the answers: lane 0 of warps 8 and 9, or a
    // whole softmax warp (whose lanes agree on it).
    int asked = 0;
    auto next_work = [&](bool &ok) {
        const int s = asked & 1;
        ok = ptx::mbar_wait(w_full(s), (asked >> 1) & 1, status);
        if (warp < 8) ok = __all_sync(0xffffffffu, ok);
        if (!ok) return -1;
        const int x = read_next(w_slot(s));
        ptx::fence_proxy_async_smem();
        if (warp < 8) __syncwarp();
        if (lane == 0) ptx::mbar_arrive(w_empty(s));
        ++asked;
        return x;
    };

    if (warp >= 8) {
        setmaxnreg_dec<88>();
        if (warp == 8 && lane == 0) {
            // ---------------- loads
            int n = 0, items = 0, issued_k = 0;
            bool ok = true;
            for (int work = blockIdx.x; ok && work >= 0; work = next_work(ok)) {
                const Span s = fwd_span(mask, args, work);
                if (s.begin() >= s.end()) continue;
                ok = ptx::mbar_wait(q_empty, (items & 1) ^ 1, status);
                if (!ok) break;
                ptx::mbar_arrive_expect_tx(q_full, 2 * F::kTile);
                for (int b = 0; b < 2; ++b)
                    for (int c = 0; c < kChunks; ++c)
                        tma_load_3d(base + F::kQ + b * F::kTile + c * kChunk, &mQ, q_full, 64 * c, s.h, s.i0 + 128 * b);
                ++items;
                for (int t = s.begin(); t < s.end(); ++t, ++n) {
                    const int st = n % kStages;
                    const uint32_t ph = (n / kStages) & 1;
                    const int j = s.first + t * kRows;
                    ok = ptx::mbar_wait(k_empty(st), ph ^ 1, status);
                    if (!ok) break;
                    ptx::mbar_arrive_expect_tx(k_full(st), F::kTile);
                    for (int c = 0; c < kChunks; ++c)
                        tma_load_3d(base + F::kK + st * F::kTile + c * kChunk, &mK, k_full(st), 64 * c, s.g, j);
                    ++issued_k;
                    ok = ptx::mbar_wait(v_empty(st), ph ^ 1, status);
                    if (!ok) break;
                    ptx::mbar_arrive_expect_tx(v_full(st), F::kTile);
                    for (int c = 0; c < kChunks; ++c)
                        tma_load_3d(base + F::kV + st * F::kTile + c * kChunk, &mV, v_full(st), 64 * c, s.g, j);
                }
            }
            // no copy may still be landing in shared memory when the block exits
            if (items) ptx::mbar_wait(q_full, (items - 1) & 1, nullptr);
            for (int i = max(issued_k - kStages, 0); i < issued_k; ++i) ptx::mbar_wait(k_full(i % kStages), (i / kStages) & 1, nullptr);
            for (int i = max(n - kStages, 0); i < n; ++i) ptx::mbar_wait(v_full(i % kStages), (i / kStages) & 1, nullptr);
        } else if (warp == 9 && lane == 0) {
            // ---------------- products
            constexpr uint32_t id_s = ptx::idesc_bf16(128, 128, false, false), id_o = ptx::idesc_bf16(128, DP, false, true);
            int n = 0, items = 0;       // key tiles and pieces of work so far
            uint32_t np[2] = {0, 0};    // products P V so far, by row block
            bool ok = true;
            for (int work = blockIdx.x; ok && work >= 0; work = next_work(ok)) {
                const Span s = fwd_span(mask, args, work);
                const int t0 = s.begin(), t1 = s.end();
                if (t0 >= t1) continue;
                ok = ptx::mbar_wait(q_full, items & 1, status);
                ++items;
                auto in = [&](int b, int t) { return b ? t >= s.b0 && t < s.b1 : t >= s.a0 && t < s.a1; };
                const uint32_t dq = desc_k(base + F::kQ), dk = desc_k(base + F::kK), dv = desc_mn(base + F::kV);
                auto score = [&](int b, int t) {  // S of row block b and tile t
                    product_features<DP>(tmem + F::kS + 128 * b, dq + b * (F::kTile >> 4), dk + ((n + t - t0) % kStages) * (F::kTile >> 4), id_s);
                    ptx::mma_commit(s_full(b));
                };
                auto wait_k = [&](int t) {
                    const int i = n + t - t0;
                    return ptx::mbar_wait(k_full(i % kStages), (i / kStages) & 1, status);
                };
                auto free_k = [&](int t) { ptx::mma_commit(k_empty((n + t - t0) % kStages)); };
                ok = ok && wait_k(t0);
                if (!ok) break;
                ptx::tc_fence_after();
                for (int b = 0; b < 2; ++b)
                    if (in(b, t0)) score(b, t0);
                free_k(t0);
                if (t0 + 1 == t1) ptx::mma_commit(q_empty);
                for (int t = t0; t < t1; ++t) {
                    const int i = n + t - t0, st = i % kStages;
                    if (t + 1 < t1) ok = wait_k(t + 1);
                    ok = ok && ptx::mbar_wait(v_full(st), (i / kStages) & 1, status);
                    if (!ok) break;
                    for (int b = 0; b < 2 && ok; ++b) {
                        if (in(b, t)) {
                            ok = ptx::mbar_wait(p_full(b), np[b] & 1, status);
                            if (!ok) break;
                            ptx::tc_fence_after();
                            const uint32_t p = tmem + F::kS + 128 * b;
                            product_tokens(tmem + F::kO + DP * b, p, p + 32, dv + st * (F::kTile >> 4), id_o, t > (b ? s.b0 : s.a0));
                            ptx::mma_commit(pv_done(b));
                            ++np[b];
                        }
                        ptx::tc_fence_after();
                        // over P, which the product above has read by then: products run in order
                        if (t + 1 < t1 && in(b, t + 1)) score(b, t + 1);
                    }
                    if (!ok) break;
                    ptx::mma_commit(v_empty(st));
                    if (t + 1 < t1) free_k(t + 1);
                    if (t + 2 == t1) ptx::mma_commit(q_empty);
                }
                n += t1 - t0;
            }
            // every product has finished before TMEM is released below: commits complete in
            // order, and the last of a piece of work is that of its last V stage
            if (n) ptx::mbar_wait(v_empty((n - 1) % kStages), ((n - 1) / kStages) & 1, nullptr);
        } else if (warp == 10 && lane == 0) {
            // ---------------- work: one answer ahead; after the first "none left" no more is asked
            for (int i = 0;; ++i) {
                const int s = i & 1;
                if (!ptx::mbar_wait(w_empty(s), ((i >> 1) & 1) ^ 1, status)) break;
                ptx::mbar_arrive_expect_tx(w_full(s), 16);
                ask_next(w_slot(s), w_full(s));
                if (!ptx::mbar_wait(w_full(s), (i >> 1) & 1, status)) break;
                if (read_next(w_slot(s)) < 0) break;
                ptx::fence_proxy_async_smem();
            }
        }
        __syncwarp();
    } else {
        // ---------------- softmax: warps 0-3 of A, 4-7 of B; thread = row
        setmaxnreg_inc<208>();
        const int b = warp / 4;
        const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
        const uint32_t tS = tmem + lanes + F::kS + 128 * b, tO = tmem + lanes + F::kO + DP * b;
        const float sl = args.a.score.scale * kLog2e;
        uint32_t ns = 0;  // score blocks so far
        bool ok = true;
        for (int work = blockIdx.x; ok && work >= 0; work = next_work(ok)) {
            const Span s = fwd_span(mask, args, work);
            const int i = s.i0 + threadIdx.x, t0 = b ? s.b0 : s.a0, t1 = b ? s.b1 : s.a1;
            const Range rg = i < mask.T ? visible(mask, i) : Range{0, 0};
            const float slope = GENERAL && args.a.score.slope ? args.a.score.slope[s.h] * kLog2e : 0.f;
            float m = -INFINITY, l = 0.f;
            for (int t = t0; t < t1; ++t) {
                const int j0 = s.first + t * kRows;
                ok = ptx::mbar_wait(s_full(b), ns & 1, status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                ptx::tc_fence_after();
                uint32_t x[128];
                __syncwarp();
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(tS + 32 * c, x + 32 * c);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < 4; ++c) pin32(x + 32 * c);
                float v[128];
                as_floats(v, x);
                if (GENERAL) {
                    // in units of log 2
#pragma unroll
                    for (int c = 0; c < 128; ++c) {
                        float y = v[c] * args.a.score.scale;
                        if (args.a.score.softcap > 0.f) y = args.a.score.softcap * tanh_exp(y * (1.f / args.a.score.softcap));
                        v[c] = fmaf(-slope, fabsf((float)(i - j0 - c)), y * kLog2e);
                    }
                }
                const int lo = rg.lo - j0, hi = rg.hi - j0;
                if (!__all_sync(0xffffffffu, lo <= 0 && hi >= kRows)) {
#pragma unroll
                    for (int c = 0; c < 128; ++c) v[c] = c >= lo && c < hi ? v[c] : -INFINITY;
                }
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < 128; c += 8)
#pragma unroll
                    for (int u = 0; u < 4; ++u) top[u] = fmaxf(top[u], fmaxf(v[c + u], v[c + 4 + u]));
                float mt = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
                if (!GENERAL) mt *= sl;
                // O and l stay relative to m until the maximum outgrows it by 2^8
                const bool grow = mt > m + 8.f || m == -INFINITY;
                if (__any_sync(0xffffffffu, grow && l > 0.f)) {
                    const float f = grow && l > 0.f ? exp2_fast(m - mt) : 1.f;
                    ok = ptx::mbar_wait(pv_done(b), (ns - 1) & 1, status);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    ptx::tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < DP; c += 32) {
                        uint32_t o[32];
                        __syncwarp();
                        tmem_ld32(tO + c, o);
                        tmem_wait_ld();
                        pin32(o);
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                        tmem_st32(tO + c, o);
                    }
                    tmem_wait_st();
                    l *= f;
                }
                if (grow) m = mt;
                const float mm = m == -INFINITY ? 0.f : m;
                uint64_t sum0 = 0, sum1 = 0;
                uint32_t pk[64];
                const uint64_t sl2 = pack2(GENERAL ? 1.f : sl, GENERAL ? 1.f : sl), m2 = pack2(-mm, -mm);
#pragma unroll
                for (int c = 0; c < 128; c += 4) {
                    float e[4];
                    unpack2(fma2(pack2(v[c], v[c + 1]), sl2, m2), e[0], e[1]);
                    unpack2(fma2(pack2(v[c + 2], v[c + 3]), sl2, m2), e[2], e[3]);
#pragma unroll
                    for (int u = 0; u < 4; ++u) e[u] = exp2_fast(e[u]);
                    sum0 = add2(sum0, pack2(e[0], e[1]));
                    sum1 = add2(sum1, pack2(e[2], e[3]));
                    pk[c / 2] = ptx::pack_bf16x2(e[0], e[1]);
                    pk[c / 2 + 1] = ptx::pack_bf16x2(e[2], e[3]);
                }
                __syncwarp();
                tmem_st32(tS, pk);
                tmem_st32(tS + 32, pk + 32);
                tmem_wait_st();
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(p_full(b));
                ++ns;
                float a0, a1, a2, a3;
                unpack2(sum0, a0, a1);
                unpack2(sum1, a2, a3);
                l += (a0 + a1) + (a2 + a3);
            }
            if (!ok) break;
            // ---------------- o and lse of this row
            const bool real = i < mask.T, none = rg.lo >= rg.hi;
            if (t1 > t0) {
                ok = ptx::mbar_wait(pv_done(b), (ns - 1) & 1, status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                ptx::tc_fence_after();
            }
            const float inv = none || !(l > 0.f) ? 0.f : 1.f / l;
            bool fine = none || isfinite(l);
            __nv_bfloat16 *out = args.a.out.at(real ? i : 0, s.h);
#pragma unroll 1
            for (int c = 0; c < DP; c += 32) {
                uint32_t o[32];
                if (t1 > t0) {
                    __syncwarp();
                    tmem_ld32(tO + c, o);
                    tmem_wait_ld();
                    pin32(o);
                }
                if (t1 <= t0 || none)
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = 0;
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    float f[8];
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        f[u] = __uint_as_float(o[e + u]) * inv;
                        fine = fine && isfinite(f[u]);
                    }
                    if (real && c + e < args.a.d)
                        *reinterpret_cast<uint4 *>(out + c + e) =
                            make_uint4(ptx::pack_bf16x2(f[0], f[1]), ptx::pack_bf16x2(f[2], f[3]), ptx::pack_bf16x2(f[4], f[5]),
                                       ptx::pack_bf16x2(f[6], f[7]));
                }
            }
            if (real) args.a.lse[(int64_t)s.h * mask.T + i] = inv > 0.f || !fine ? (m + log2f(l)) * kLn2 : -INFINITY;
            // rows that masked infinities or NaN have reached
            uint32_t bad = __ballot_sync(0xffffffffu, real && !fine);
            __syncwarp();
            for (; bad; bad &= bad - 1) row_fwd(args.a, i - lane + __ffs(bad) - 1, s.h, lane);
        }
    }

    ptx::tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, 512);
    }
}

}  // namespace tc
}  // namespace attn
}  // namespace noble
