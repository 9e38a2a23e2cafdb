// Forward attention over documents on the tensor cores.
//
// A piece of work is 256 queries of one head, as two row blocks A and B of 128, over the
// key tiles that they see:
//     S = Q K^T        operands in shared memory, S in TMEM
//     P = exp2(S - m)  one thread per row; P (bf16) over S in TMEM
//     O += P V         P from TMEM, V MN-major in shared memory
// Row blocks alternate on the tensor pipe: while one's warps compute P the pipe works on
// the other's products, and each key tile is read from L2 once for 256 queries (32 bytes
// per clock and SM at the full rate).  Score blocks go to as many buffers as TMEM has room
// for beside O, three with heads of 64 features, so that S is there before its warps are.
// O stays in TMEM; it is scaled down only when a row's
// maximum has grown by more than 2^8 since the last time, which after the first tiles
// happens rarely.  Sums and maxima are fp32; P is rounded to bf16 for the product (each
// to 2^-9 of itself), its sum is that of the unrounded values.
//
// What bounds it: with heads of 128 features the tensor pipe (16384 tokens, 16 heads: 1383 us
// with all seen, 700 causal, 1590 and 1571 TFLOP/s), with 64 the exponentials (1007 us, 1092
// TFLOP/s).  Short documents pay for each piece's start, masked tiles and rows written (8 of 1024
// tokens, 16 heads of 64: 41 us, 64 of 197, 12 heads: 46), capped scores for their tanh on the
// FMA pipe (7001 tokens, 16 heads on 4 of 128: 110 us, 69 without a cap).
#pragma once

#include "attn_tc.cuh"

namespace noble {
namespace attn {
namespace tc {

template <int DP>
struct Fwd {
    static constexpr int kThreads = 384;  // two softmax warpgroups; loading, product, work and padding warps
    static constexpr int kStages = DP == 64 ? 4 : 2;
    static constexpr int kBuffers = DP == 64 ? 3 : 2;  // of 128 TMEM columns for S
    static constexpr uint32_t kTile = kChunk * (DP / 64);
    static constexpr uint32_t kQ = 0, kK = 2 * kTile, kV = kK + kStages * kTile, kDocs = kV + kStages * kTile;
    static constexpr uint32_t kWork = kDocs + 2 * kDocsInSmem * 4, kBars = kWork + Work::kBytes;
    // q full/empty; k and v full/empty by stage; s full by row block and its own count of
    // score blocks (a phase of another's would be taken for one of its own); p full by
    // buffer; pv done by row block; k and v with padding landed by stage
    static constexpr int kNumBars = 2 + 4 * kStages + 3 * kBuffers + 2 + 2 * kStages;
    static constexpr uint32_t kAgain = kBars + 8 * kNumBars + 16;
    static constexpr uint32_t kBytes = kAgain + Again::kBytes;
    static constexpr uint32_t kDynamic = kBytes + 1024;
    static constexpr uint32_t kO = 128 * kBuffers;  // TMEM column of O
};

struct FwdArgs {
    RowArgs<__nv_bfloat16> a;
    int tiles;  // of 256 queries
    uint32_t *status;
};

// Key tiles of a row block, counted from the first key that its piece of work sees: A
// has the tiles [0, a1), B [b0, b1), with none in between that neither has.
struct Span {
    int i0, h, g, first, a1, b0, b1;
    __device__ __forceinline__ int end() const { return max(a1, b1); }
    __device__ __forceinline__ bool in(int b, int t) const { return b ? t >= b0 && t < b1 : t < a1; }
    // score blocks before that of (t, b), in the order A, B of a tile
    __device__ __forceinline__ int before(int t, int b) const { return min(t + b, a1) + clampi(t, b0, b1) - b0; }
};
__device__ __forceinline__ Span as_span(const Piece &p) { return {p.v[0], p.v[1], p.v[2], p.v[3], p.v[4], p.v[5], p.v[6]}; }

__device__ __forceinline__ Piece fwd_piece(const Mask &m, const FwdArgs &f, int work)
{
    const int h = work % f.a.n_q, i0 = (f.tiles - 1 - work / f.a.n_q) * 256;
    const int first = visible(m, i0).lo;
    int a1 = (max(visible(m, min(i0 + 127, m.T - 1)).hi - first, 0) + kRows - 1) / kRows, b0 = a1, b1 = a1;
    if (i0 + 128 < m.T) {
        b0 = max(visible(m, i0 + 128).lo - first, 0) / kRows;  // below 0 only if the documents' starts do not ascend
        b1 = (max(visible(m, min(i0 + 255, m.T - 1)).hi - first, 0) + kRows - 1) / kRows;
        if (b1 <= b0) b0 = b1 = a1;
        else a1 = max(a1, b0);
    }
    return {{i0, h, h / (f.a.n_q / f.a.n_kv), first, a1, b0, b1, 0}};
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
    auto s_full = [&](int b, int i) { return bars + 8u * (2 + 4 * kStages + b * F::kBuffers + i); };
    auto p_full = [&](int i) { return bars + 8u * (2 + 4 * kStages + 2 * F::kBuffers + i); };
    auto pv_done = [&](int b) { return bars + 8u * (2 + 4 * kStages + 3 * F::kBuffers + b); };
    Padding pad_k{bars + 8u * (4 + 4 * kStages + 3 * F::kBuffers), 0}, pad_v{pad_k.at(kStages), 0};
    const Work works{base + F::kWork};
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + F::kBars + 8 * F::kNumBars);
    const Again again{reinterpret_cast<uint32_t *>(smem + F::kAgain)};
    const int warp = (int)uniform(threadIdx.x / 32), lane = threadIdx.x % 32;
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
            ptx::mbar_init(pad_k.at(s), 1);
            ptx::mbar_init(pad_v.at(s), 1);
        }
        for (int i = 0; i < F::kBuffers; ++i) {
            ptx::mbar_init(s_full(0, i), 1);
            ptx::mbar_init(s_full(1, i), 1);
            ptx::mbar_init(p_full(i), 4);
        }
        for (int b = 0; b < 2; ++b) ptx::mbar_init(pv_done(b), 1);
        works.init(11);
        ptx::fence_barrier_init();
    }
    if (warp == 9) {
        ptx::tmem_alloc(ptx::smem_u32(tmem_slot), 512);
        ptx::tmem_relinquish();
    }
    again.init();
    const Mask mask = mask_in_smem<kDocsInSmem>(args.a.mask, reinterpret_cast<int32_t *>(smem + F::kDocs));
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = uniform(*tmem_slot);

    Piece pc;
    if (warp >= 8) {
        setmaxnreg_dec<88>();
        const int padding = padding_from(mask);
        auto padded = [&](const Span &s) { return s.first + s.end() * kRows > padding; };  // its last tile
        if (warp == 8 && lane == 0) {
            // ---------------- loads
            int n = 0, items = 0, issued_k = 0;
            bool ok = true;
            for (int w = 0; ok && works.take(pc, w, false, true, 0, status); ++w) {
                const Span s = as_span(pc);
                if (s.end() == 0) continue;
                ok = ptx::mbar_wait(q_empty, (items & 1) ^ 1, status);
                if (!ok) break;
                ptx::mbar_arrive_expect_tx(q_full, 2 * F::kTile);
                for (int b = 0; b < 2; ++b)
                    for (int c = 0; c < kChunks; ++c)
                        tma_load_3d(base + F::kQ + b * F::kTile + c * kChunk, &mQ, q_full, 64 * c, s.h, s.i0 + 128 * b);
                ++items;
                for (int t = 0; t < s.end(); ++t, ++n) {
                    const int st = n % kStages;
                    const uint32_t ph = (n / kStages) & 1;
                    const int j = s.first + t * kRows;
                    ok = ptx::mbar_wait(k_empty(st), ph ^ 1, status);
                    if (!ok) break;
                    const bool pad = t + 1 == s.end() && padded(s);
                    const uint32_t to_k = pad ? pad_k.at(st) : k_full(st), to_v = pad ? pad_v.at(st) : v_full(st);
                    ptx::mbar_arrive_expect_tx(to_k, F::kTile);
                    for (int c = 0; c < kChunks; ++c)
                        tma_load_3d(base + F::kK + st * F::kTile + c * kChunk, &mK, to_k, 64 * c, s.g, j);
                    ++issued_k;
                    ok = ptx::mbar_wait(v_empty(st), ph ^ 1, status);
                    if (!ok) break;
                    ptx::mbar_arrive_expect_tx(to_v, F::kTile);
                    for (int c = 0; c < kChunks; ++c)
                        tma_load_3d(base + F::kV + st * F::kTile + c * kChunk, &mV, to_v, 64 * c, s.g, j);
                }
            }
            // no copy may still be landing in shared memory when the block exits
            if (items) ptx::mbar_wait(q_full, (items - 1) & 1, nullptr);
            for (int i = max(issued_k - kStages, 0); i < issued_k; ++i) ptx::mbar_wait(k_full(i % kStages), (i / kStages) & 1, nullptr);
            for (int i = max(n - kStages, 0); i < n; ++i) ptx::mbar_wait(v_full(i % kStages), (i / kStages) & 1, nullptr);
        } else if (warp == 9) {
            // ---------------- products
            const bool leader = elect_one();
            constexpr uint32_t id_s = ptx::idesc_bf16(128, 128, false, false), id_o = ptx::idesc_bf16(128, DP, false, true);
            const uint32_t dq = desc_k(base + F::kQ), dk = desc_k(base + F::kK), dv = desc_mn(base + F::kV);
            // Rings by index and parity, moved on without a division.
            constexpr uint32_t kStep = F::kTile >> 4;
            int items = 0;
            uint32_t last = 0;                // the stage of the last key tile
            uint32_t st_s = 0, ph_s = 0;      // stage of the next S
            uint32_t st_v = 0, ph_v = 0;      // of the next P V
            uint32_t buf_s = 0, buf_p = 0, ph_p = 0;  // score buffers of both
            uint32_t of0 = 0, of1 = 0;        // the next s_full of A and of B
            auto next = [](uint32_t i, uint32_t n) { return i + 1 == n ? 0u : i + 1; };
            bool ok = true;
            for (int w = 0; ok && works.take(pc, w, true, false, lane, status); ++w) {
                const Span s = as_span(pc);
                const int t1 = s.end();
                if (t1 == 0) continue;
                ok = wait_warp(q_full, items & 1, status);
                ++items;
                int ts = 0;  // tile and row block of the next S
                bool to_b = s.a1 == 0;
                auto score = [&] {
                    if (!to_b) {
                        if (!wait_warp(k_full(st_s), ph_s, status)) return false;
                        ptx::tc_fence_after();
                        if (leader) {
                            product_features<DP>(tmem + 128 * buf_s, dq, dk + st_s * kStep, id_s);
                            ptx::mma_commit(s_full(0, of0));
                        }
                        of0 = next(of0, F::kBuffers), buf_s = next(buf_s, F::kBuffers);
                        if (ts >= s.b0 && ts < s.b1) {
                            to_b = true;
                            return true;
                        }
                    } else {
                        if (ts >= s.a1 && !wait_warp(k_full(st_s), ph_s, status)) return false;
                        ptx::tc_fence_after();
                        if (leader) {
                            product_features<DP>(tmem + 128 * buf_s, dq + kStep, dk + st_s * kStep, id_s);
                            ptx::mma_commit(s_full(1, of1));
                        }
                        of1 = next(of1, F::kBuffers), buf_s = next(buf_s, F::kBuffers);
                    }
                    if (leader) ptx::mma_commit(k_empty(st_s));
                    st_s = next(st_s, kStages), ph_s ^= st_s == 0;
                    ++ts;
                    to_b = ts >= s.a1;
                    if (ts == t1 && leader) ptx::mma_commit(q_empty);  // the last use of Q
                    return true;
                };
                // P V of one row block; its buffer is then the next S's: products run in order
                auto weigh = [&](uint32_t o, bool more, uint32_t done) {
                    if (!wait_warp(p_full(buf_p), ph_p, status)) return false;
                    ptx::tc_fence_after();
                    const uint32_t p = tmem + 128 * buf_p;
                    if (leader) {
                        product_tokens(o, p, p + 32, dv + st_v * kStep, id_o, more);
                        ptx::mma_commit(done);
                    }
                    buf_p = next(buf_p, F::kBuffers), ph_p ^= buf_p == 0;
                    return ts == t1 || score();
                };
                for (int i = 0; ok && i < F::kBuffers && ts < t1; ++i) ok = score();
                for (int t = 0; ok && t < t1; ++t) {
                    ok = wait_warp(v_full(st_v), ph_v, status);
                    if (ok && t < s.a1) ok = weigh(tmem + F::kO, t > 0, pv_done(0));
                    if (ok && t >= s.b0 && t < s.b1) ok = weigh(tmem + F::kO + DP, t > s.b0, pv_done(1));
                    if (leader) ptx::mma_commit(v_empty(st_v));
                    last = 2 * st_v + ph_v + 1;
                    st_v = next(st_v, kStages), ph_v ^= st_v == 0;
                }
            }
            // every product has finished before TMEM is released below: commits complete in
            // order, and the last of a piece of work is that of its last V stage
            if (last) wait_warp(v_empty((last - 1) / 2), (last - 1) & 1, nullptr);
        } else if (warp == 10 && lane == 0) {
            works.hand_out([&](int work) { return fwd_piece(mask, args, work); }, again.any(), status);
        } else if (warp == 11) {
            // ---------------- padding
            int n = 0;
            for (int w = 0; works.take(pc, w, true, false, lane, status); ++w) {
                const Span s = as_span(pc);
                n += s.end();
                if (s.end() == 0 || !padded(s)) continue;
                const int st = (n - 1) % kStages, from = padding - (s.first + (s.end() - 1) * kRows);
                if (!pad_k.clear<DP>(smem + F::kK + st * F::kTile, st, from, k_full(st), lane, status)) break;
                if (!pad_v.clear<DP>(smem + F::kV + st * F::kTile, st, from, v_full(st), lane, status)) break;
            }
        }
        __syncwarp();
    } else {
        // ---------------- softmax: warps 0-3 of A, 4-7 of B; thread = row
        setmaxnreg_inc<208>();
        const int b = warp / 4;
        const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
        const uint32_t tO = tmem + lanes + F::kO + DP * b;
        const float sl = args.a.score.scale * kLog2e;
        uint32_t ns = 0;  // score blocks so far: of this row block
        int all = 0;      // and of both
        bool ok = true;
        for (int w = 0; ok && works.take(pc, w, true, false, lane, status); ++w) {
            const Span s = as_span(pc);
            const int i = s.i0 + threadIdx.x, t0 = b ? s.b0 : 0, t1 = b ? s.b1 : s.a1;
            const Range rg = i < mask.T ? visible(mask, i) : Range{0, 0};
            const float slope = GENERAL && args.a.score.slope ? args.a.score.slope[s.h] * kLog2e : 0.f;
            float m = -INFINITY, l = 0.f;
            for (int t = t0; t < t1; ++t) {
                const int j0 = s.first + t * kRows;
                const int nth = all + s.before(t, b);
                const int buf = nth % F::kBuffers;
                const uint32_t tS = tmem + lanes + 128 * buf;
                ok = ptx::mbar_wait(s_full(b, ns % F::kBuffers), (ns / F::kBuffers) & 1, status);
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
                    uint32_t none[1];
                    general_scores<128, false>(v, none, args.a.score, slope, (float)(i - j0), rg.lo < rg.hi);
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
                // one product P V of a row block at a time is outstanding, so that a phase of
                // pv_done is never mistaken for the one before; by now it is done
                if (ns > 0) {
                    ok = ptx::mbar_wait(pv_done(b), (ns - 1) & 1, status);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                }
                __syncwarp();
                tmem_st32(tS, pk);
                tmem_st32(tS + 32, pk + 32);
                tmem_wait_st();
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(p_full(buf));
                ++ns;
                float a0, a1, a2, a3;
                unpack2(sum0, a0, a1);
                unpack2(sum1, a2, a3);
                l += (a0 + a1) + (a2 + a3);
            }
            if (!ok) break;
            all += s.a1 + s.b1 - s.b0;
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
            __nv_bfloat16 *out = args.a.out.at(i - lane, s.h);
#pragma unroll 1
            for (int c = 0; c < DP; c += 32) {
                uint32_t o[32];
                if (t1 > t0) {
                    __syncwarp();
                    tmem_ld32(tO + c, o);
                    tmem_wait_ld();
                    pin32(o);
                }
                fine &= write_rows(o, inv, t1 <= t0 || none, out + c, args.a.out.row, mask.T - (i - lane), args.a.d - c, lane);
            }
            if (real) args.a.lse[(int64_t)s.h * mask.T + i] = inv > 0.f || !fine ? (m + log2f(l)) * kLn2 : -INFINITY;
            // rows that masked infinities or NaN have reached
            again.note(warp, lane, i - lane, s.h, __ballot_sync(0xffffffffu, real && !fine));
        }
        again.each(warp, [&](int, int i, int h) { row_fwd(args.a, i, h, lane); });
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
