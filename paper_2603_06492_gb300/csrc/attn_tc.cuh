// Attention over documents on the tensor cores: what forward and backward share.
//
// Tiles are 128 tokens by 64 features of bf16 with the 128-byte swizzle (16 KB, one
// TMA box), so the same tile serves as a K-major operand (features contracted) and as
// an MN-major one (tokens contracted).  Heads of 65 to 128 features take two tiles;
// TMA fills features past d and tokens past T with zeros.
//
// TMEM lanes are rows of a score block: a thread of the four warps of a warpgroup owns
// one row, so that a softmax needs no exchange between threads.
#pragma once

#include <cuda_fp16.h>
#include <type_traits>

#include "attn_mask.cuh"
#include "sm100_ptx.cuh"

namespace noble {
namespace attn {
namespace tc {

constexpr int kRows = 128;                  // rows of a score block, keys of a tile
constexpr uint32_t kChunk = 128 * 64 * 2;   // bytes of a tile of 64 features
constexpr int kDocsInSmem = 1024;           // document starts kept in shared memory

// ---------------------------------------------------------------- PTX
// 3-D tiled load (features, head, token); c0 a multiple of 8 elements.
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1, int c2)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}

// One lane of the warp, always the same.
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}\n" : "=r"(p));
    return p != 0;
}
// A value that all lanes have, as one that the compiler knows they have.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(0xffffffffu, v, 0); }

// Products are issued by one lane of a warp whose lanes otherwise stay together: operands
// then are in uniform registers, which a product reads, and not moved there one by one
// (65 clocks for each, as many as the tensor pipe takes for 128 columns).  Descriptors
// are made of a low word per operand, to which a constant is added per step, and a
// high word that all share (128-byte swizzle, 1024 bytes between groups of 8 rows).
constexpr uint32_t kDescHigh = 64u | (1u << 14) | (2u << 29);
// K-major operand of a token tile (features contracted), MN-major one (tokens contracted)
__device__ __forceinline__ uint32_t desc_k(uint32_t tile) { return ((tile & 0x3FFFFu) >> 4) | (1u << 16); }
__device__ __forceinline__ uint32_t desc_mn(uint32_t tile) { return ((tile & 0x3FFFFu) >> 4) | ((kChunk >> 4) << 16); }
__host__ __device__ constexpr uint32_t step_k(int kk) { return ((kk >> 2) * kChunk + (kk & 3) * 32) >> 4; }
__host__ __device__ constexpr uint32_t step_mn(int kk) { return kk * 2048 >> 4; }

__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}\n" ::"r"(d_tmem),
        "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "r"(kDescHigh)
        : "memory");
}
// A from TMEM, two bf16 per 32-bit column, K ascending.
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 db, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}\n" ::"r"(d_tmem),
        "r"(a_tmem), "r"(b), "r"(idesc), "r"(accumulate), "r"(kDescHigh)
        : "memory");
}
// A bounded wait of a whole warp: the same answer in all lanes.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, uint32_t *status)
{
    return __all_sync(0xffffffffu, ptx::mbar_wait(bar, parity, status));
}
// D = A B^T over the features of two token tiles (DP of them)
template <int DP>
__device__ __forceinline__ void product_features(uint32_t d_tmem, uint32_t a, uint32_t b, uint32_t idesc)
{
#pragma unroll
    for (int kk = 0; kk < DP / 16; ++kk) mma_ss(d_tmem, a + step_k(kk), b + step_k(kk), idesc, kk > 0);
}
// D (+)= A B over 128 tokens, A at two places of 64 tokens each in TMEM
__device__ __forceinline__ void product_tokens(uint32_t d_tmem, uint32_t a_low, uint32_t a_high, uint32_t b, uint32_t idesc, bool more)
{
#pragma unroll
    for (int kk = 0; kk < kRows / 16; ++kk)
        mma_ts(d_tmem, (kk < 4 ? a_low : a_high) + 8 * (kk & 3), b + step_mn(kk), idesc, kk > 0 ? 1u : (uint32_t)more);
}

// 32 columns of this thread's TMEM lane; valid only after tmem_wait_ld.  These and the
// stores below are for whole warps: after code whose lanes may have parted (a wait, a
// masked score) a __syncwarp comes before them.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t *r)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
// Waits for this thread's TMEM loads.  The values loaded pass through pin32 after
// it, so that no use of them is moved before the wait.
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pin32(uint32_t *r)
{
    asm volatile(""
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]));
    asm volatile(""
                 : "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                   "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31]));
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t *r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

template <int N>
__device__ __forceinline__ void as_floats(float (&f)[N], const uint32_t (&r)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = __uint_as_float(r[i]);
}

// 32 fp32 features of a warp's 32 rows, a row per lane, times f, to rows of bf16 in memory;
// zeros where `zero`.  Lanes exchange pieces of 16 bytes in fours, so that four of
// them write 64 bytes of a row: a store whose lanes all have rows of their own takes the 32
// clocks of 32 lines (64 images of 197 tokens, 12 heads of 64: the backward 145 us so, 129
// with the exchange).
// Returns whether the row is finite.  All lanes call it together; `out`: row of lane 0.
__device__ __forceinline__ bool write_rows(const uint32_t (&o)[32], float f, bool zero, __nv_bfloat16 *out, int64_t stride,
                                           int rows, int cols, int lane)
{
    uint32_t w[16];
    uint64_t left = 0;  // stays 0 unless something is infinite or NaN
    const uint64_t f2 = pack2(f, f);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint64_t x = mul2(pack2(__uint_as_float(o[2 * i]), __uint_as_float(o[2 * i + 1])), f2);
        left = fma2(x, 0ull, left);
        float a, b;
        unpack2(x, a, b);
        w[i] = zero ? 0u : ptx::pack_bf16x2(a, b);
    }
    // piece c of lane l's row goes to lane c of the four, as its piece l
#pragma unroll
    for (int bit = 1; bit < 4; bit <<= 1)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if (c & bit) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t &lo = w[4 * c + i], &hi = w[4 * (c | bit) + i];
                const uint32_t got = __shfl_xor_sync(0xffffffffu, lane & bit ? lo : hi, bit);
                if (lane & bit) lo = got;
                else hi = got;
            }
        }
    const int first = lane & ~3, col = (lane & 3) * 8;
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (first + r < rows && col < cols)
            *reinterpret_cast<uint4 *>(out + (first + r) * stride + col) = make_uint4(w[4 * r], w[4 * r + 1], w[4 * r + 2], w[4 * r + 3]);
    return zero || sum2(left) == 0.f;
}

// The last tile of the last document may reach into padding, the tokens behind all documents, which
// hold anything, infinities and NaN too.  Such a tile is loaded to a barrier of its own; a warp
// that has little else to do clears its padding rows when it has landed and then arrives
// on the barrier that the products wait for: these know nothing of it (checks among their waits
// cost 16384 tokens of 64 features 5 % forward, 3 % backward).  Other tokens that a tile holds and a row does
// not see belong to a document, and are finite unless something went wrong: see row_fwd.
__device__ __forceinline__ int padding_from(const Mask &m) { const int end = docs_end(m); return end < m.T ? end : INT32_MAX; }
// Barriers `landed` + 8 st by stage, in use for tiles with padding only: parities by stage.
struct Padding {
    uint32_t landed, parities;
    __device__ __forceinline__ uint32_t at(int st) const { return landed + 8u * st; }
    // A whole warp: rows `from` and on of the tile of stage st.
    template <int DP>
    __device__ __forceinline__ bool clear(uint8_t *tile, int st, int from, uint32_t full, int lane, uint32_t *status)
    {
        if (!wait_warp(at(st), parities >> st & 1, status)) return false;
        parities ^= 1u << st;
#pragma unroll
        for (int c = 0; c < DP / 64; ++c)
            for (int x = 8 * max(from, 0) + lane; x < 8 * kRows; x += 32) *reinterpret_cast<uint4 *>(tile + c * kChunk + 16 * x) = make_uint4(0, 0, 0, 0);
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(full);
        return true;
    }
};

// Scores of N columns of a row in units of log 2, from q.k: capped, and biased by the
// distance `far` - column of query and key; gs their derivatives by scale q.k as pairs
// of 16-bit floats, for a product that is rounded to 8 bits.  Nothing here converts an
// integer per column, which would run beside the exponentials at their rate.
//
// tanh takes an exponential and a reciprocal, which with the softmax's own exponential
// make the special function unit the limit.  Where all of a warp's arguments are within
// 0.6 its Taylor series to x^15 does, within 0.33 that to x^9: the first term left out,
// 6e-4 x^17 and 9e-3 x^11, is at most 2e-7 of the result.  Ragged documents of 7001 tokens,
// 16 + 4 heads of 128, cap 30: forward 136 us without series, 125 with the longer one, 113
// with both.
enum : int { kNoCap = 0, kCapShort = 1, kCapSeries = 2, kCapExact = 3 };
struct Capping {
    float in, out;  // kNoCap: s = out q.k
    int mode;
};
// seen: whether the row sees anything; if not, its scores have no part in the choice.
template <int N>
__device__ __forceinline__ Capping capping(const float (&x)[N], const Score &sc, bool seen)
{
    if (!(sc.softcap > 0.f)) return {0.f, sc.scale * kLog2e, kNoCap};
    const float in = sc.scale / sc.softcap;
    float top[4] = {};
#pragma unroll
    for (int c = 0; c < N; c += 4)
#pragma unroll
        for (int u = 0; u < 4; ++u) top[u] = fmaxf(top[u], fabsf(x[c + u]));
    const float most = seen ? fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * fabsf(in) : 0.f;
    const int mode = __all_sync(0xffffffffu, most < 0.33f) ? kCapShort : __all_sync(0xffffffffu, most < 0.6f) ? kCapSeries : kCapExact;
    return {in, sc.softcap * kLog2e, mode};
}
// Two scores, in place, and their derivatives.
template <int MODE, bool GRAD>
__device__ __forceinline__ void cap_pair(uint64_t &x, uint64_t &g, const Capping &cap)
{
    const uint64_t one2 = pack2(1.f, 1.f), minus2 = pack2(-1.f, -1.f), out2 = pack2(cap.out, cap.out);
    if (MODE == kNoCap) {
        x = mul2(x, out2);
        if (GRAD) g = one2;
    } else if (MODE != kCapExact) {
        constexpr int kTerms = MODE == kCapShort ? 4 : 7;
        const float k[7] = {-1.f / 3.f, 2.f / 15.f, -17.f / 315.f, 62.f / 2835.f, -1382.f / 155925.f, 21844.f / 6081075.f,
                            -929569.f / 638512875.f};
        const uint64_t a = mul2(x, pack2(cap.in, cap.in)), u = mul2(a, a);
        uint64_t p = pack2(k[kTerms - 1], k[kTerms - 1]);
#pragma unroll
        for (int e = kTerms - 2; e >= 0; --e) p = fma2(p, u, pack2(k[e], k[e]));
        const uint64_t t = mul2(a, fma2(p, u, one2));
        x = mul2(t, out2);
        if (GRAD) g = fma2(mul2(t, minus2), t, one2);
    } else {
        float a, b;
        unpack2(mul2(x, pack2(cap.in, cap.in)), a, b);
        const uint64_t t = pack2(tanh_exp(a), tanh_exp(b));
        x = mul2(t, out2);
        if (GRAD) g = fma2(mul2(t, minus2), t, one2);
    }
}
// f(MODE) for the mode of a Capping
template <class F>
__device__ __forceinline__ void with_cap(int mode, F &&f)
{
    if (mode == kNoCap) f(std::integral_constant<int, kNoCap>{});
    else if (mode == kCapShort) f(std::integral_constant<int, kCapShort>{});
    else if (mode == kCapSeries) f(std::integral_constant<int, kCapSeries>{});
    else f(std::integral_constant<int, kCapExact>{});
}
template <int N, bool GRAD>
__device__ __forceinline__ void general_scores(float (&x)[N], uint32_t (&gs)[GRAD ? N / 2 : 1], const Score &sc, float slope, float far, bool seen)
{
    const Capping cap = capping(x, sc, seen);
    with_cap(cap.mode, [&](auto mode) {
#pragma unroll
        for (int c = 0; c < N; c += 2) {
            uint64_t v = pack2(x[c], x[c + 1]), g = 0;
            cap_pair<mode.value, GRAD>(v, g, cap);
            unpack2(v, x[c], x[c + 1]);
            if (GRAD) {
                float a, b;
                unpack2(g, a, b);
                const __half2 h = __floats2half2_rn(a, b);
                gs[GRAD ? c / 2 : 0] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
    });
    if (sc.slope) {
#pragma unroll
        for (int c = 0; c < N; ++c) x[c] = fmaf(-slope, fabsf(far - (float)c), x[c]);
    }
}

template <int N>
__device__ __forceinline__ void setmaxnreg_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void setmaxnreg_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// ---------------------------------------------------------------- rows computed again
// Rows that come out not finite (row_fwd and its like say why) are noted while a block's pieces of
// work run and computed again when the block is through with them: one such row of a
// long document takes milliseconds, many take longer than the other warps' waits last.  A block
// that has noted rows asks for no further piece, and the launch starts another one for what is
// left.  So a warp notes rows of at most 7 pieces: those of piece w when it has taken w + 1 at most;
// w + 5 would be asked for only after it has taken w + 2; and no warp is behind w - 2.
struct Again {
    static constexpr int kPieces = 8, kWarps = 8;
    static constexpr uint32_t kBytes = 4 * (1 + kWarps + 2 * kWarps * kPieces) + 4;
    uint32_t *mem;  // whether any rows are noted; pieces noted per warp; (first row of 32 and head, rows) of each
    __device__ __forceinline__ volatile uint32_t *any() const { return mem; }
    __device__ __forceinline__ void init() const  // all threads, before a __syncthreads
    {
        if (threadIdx.x <= kWarps) mem[threadIdx.x] = 0;
    }
    // The warp's `rows` of row0 (a multiple of 32) and on, of a head; all lanes together.
    __device__ __forceinline__ void note(int warp, int lane, int row0, int head, uint32_t rows) const
    {
        if (rows && lane == 0) {
            uint32_t *at = mem + 1 + kWarps + 2 * (warp * kPieces + mem[1 + warp]++);
            at[0] = (uint32_t)row0 >> 5 | (uint32_t)head << 19, at[1] = rows;
            *any() = 1;
        }
        __syncwarp();
    }
    // f(warp that noted it, row, head) for every row noted, by the warps in turn, all of which call
    // this when they have no more to note.
    template <class F>
    __device__ __forceinline__ void each(int warp, F &&f) const
    {
        __syncwarp();
        asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory");
        if (!*any()) return;
        int k = 0;
        for (int w = 0; w < kWarps; ++w)
            for (uint32_t e = 0; e < mem[1 + w]; ++e) {
                const uint32_t *at = mem + 1 + kWarps + 2 * (w * kPieces + e);
                for (uint32_t rows = at[1]; rows; rows &= rows - 1)
                    if (k++ % kWarps == warp) f(w, (int)((at[0] & 0x7ffffu) << 5) + __ffs(rows) - 1, (int)(at[0] >> 19));
            }
    }
};

// ---------------------------------------------------------------- work handed out by the launch
// A block that has finished its piece of work takes over that of a block of the grid
// that has not started (cluster launch control), so that blocks set up once and
// pieces of unequal size balance.  One thread asks, works out what the piece is and
// publishes that in one of two slots of shared memory, a piece ahead of its readers:
// it asks again when the loading thread has taken the last one.
__device__ __forceinline__ void ask_next(uint32_t slot, uint32_t bar)
{
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(slot),
                 "r"(bar)
                 : "memory");
}
// The block's index of the answer in `slot`, or -1 if there was none left.
__device__ __forceinline__ int read_next(uint32_t slot)
{
    int x;
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b128 h;\n\t.reg .b32 y, z, w;\n\t"
        "ld.shared.b128 h, [%1];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n\t"
        "mov.b32 %0, -1;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%0, y, z, w}, h;\n\t}\n"
        : "=r"(x)
        : "r"(slot)
        : "memory");
    return x;
}

struct Piece {
    int v[8];  // v[0] < 0: none left
};
struct Work {
    uint32_t mem;  // 6 barriers (answer, taken, full and empty by slot), the answer, two pieces
    static constexpr uint32_t kBytes = 48 + 16 + 2 * 32;
    __device__ __forceinline__ uint32_t answered() const { return mem; }
    __device__ __forceinline__ uint32_t taken() const { return mem + 8; }
    __device__ __forceinline__ uint32_t full(int s) const { return mem + 16 + 8 * s; }
    __device__ __forceinline__ uint32_t empty(int s) const { return mem + 32 + 8 * s; }
    __device__ __forceinline__ uint32_t answer() const { return mem + 48; }
    __device__ __forceinline__ uint32_t slot(int s) const { return mem + 64 + 32 * s; }
    __device__ __forceinline__ void init(int readers) const
    {
        ptx::mbar_init(answered(), 1);
        ptx::mbar_init(taken(), 1);
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(full(s), 1);
            ptx::mbar_init(empty(s), readers);
        }
    }
    // The thread that hands out; describe(index) is the piece of a block.  It asks for no more once
    // `enough` is set.
    template <class F>
    __device__ __forceinline__ void hand_out(F &&describe, volatile uint32_t *enough, uint32_t *status) const
    {
        int work = blockIdx.x;
        for (int k = 0;; ++k) {
            Piece p;
            if (work >= 0) p = describe(work);
            else p.v[0] = -1;
            const uint32_t at = slot(k & 1);
            if (!ptx::mbar_wait(empty(k & 1), ((k >> 1) & 1) ^ 1, status)) break;
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(p.v[0]), "r"(p.v[1]), "r"(p.v[2]), "r"(p.v[3]) : "memory");
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + 16), "r"(p.v[4]), "r"(p.v[5]), "r"(p.v[6]), "r"(p.v[7]) : "memory");
            ptx::mbar_arrive(full(k & 1));
            if (work < 0) break;  // no more is asked after the first "none left"
            if (!ptx::mbar_wait(taken(), k & 1, status)) break;
            if (*enough) {
                work = -1;
                continue;
            }
            ptx::mbar_arrive_expect_tx(answered(), 16);
            ask_next(answer(), answered());
            if (!ptx::mbar_wait(answered(), k & 1, status)) break;
            work = read_next(answer());
            ptx::fence_proxy_async_smem();
        }
    }
    // Piece k for a reader, `whole` warps together; false when there is none left.
    __device__ __forceinline__ bool take(Piece &p, int k, bool whole, bool loader, int lane, uint32_t *status) const
    {
        bool ok = ptx::mbar_wait(full(k & 1), (k >> 1) & 1, status);
        if (whole) ok = __all_sync(0xffffffffu, ok);
        if (!ok) return false;
        const uint32_t at = slot(k & 1);
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(p.v[0]), "=r"(p.v[1]), "=r"(p.v[2]), "=r"(p.v[3]) : "r"(at) : "memory");
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(p.v[4]), "=r"(p.v[5]), "=r"(p.v[6]), "=r"(p.v[7]) : "r"(at + 16) : "memory");
        if (whole) {
#pragma unroll
            for (int i = 0; i < 8; ++i) p.v[i] = (int)uniform((uint32_t)p.v[i]);
        }
        if (lane == 0) ptx::mbar_arrive(empty(k & 1));
        if (loader && p.v[0] >= 0) ptx::mbar_arrive(taken());
        return p.v[0] >= 0;
    }
};

// The document starts (and prefixes) in shared memory where they fit, since every
// piece of work searches them; call with all threads, before a __syncthreads.
template <int KEPT>
__device__ __forceinline__ Mask mask_in_smem(const Mask &m, int32_t *sm)
{
    Mask r = m;
    if (m.n_docs >= KEPT) return r;
    for (int i = threadIdx.x; i <= m.n_docs; i += blockDim.x) sm[i] = m.doc_start[i];
    r.doc_start = sm;
    if (m.prefix) {
        for (int i = threadIdx.x; i < m.n_docs; i += blockDim.x) sm[KEPT + i] = m.prefix[i];
        r.prefix = sm + KEPT;
    }
    return r;
}

}  // namespace tc
}  // namespace attn
}  // namespace noble
