// C-ABI entry points of the attention operators (declared in include/noble.h): rotary
// positions, the paged cache, attention over documents and over the cache.
//
// Host side only: argument checks, workspaces and kernel dispatch.
#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <limits>

#include "host.cuh"
#include "attn_mask.cuh"
#include "attn_paged.cuh"
#include "attn_paged_mma.cuh"
#include "attn_simt.cuh"
#include "attn_tc_bwd.cuh"
#include "attn_tc_fwd.cuh"
#include "rope.cuh"

namespace noble {
namespace {

using bf = __nv_bfloat16;
constexpr int kSms = 152;  // of a GB300; rules that choose between orders of sums take this, not the device's

noble_status heads_count(int64_t n_q, int64_t n_kv)
{
    if (n_q < 1 || n_kv < 1 || n_q > 4096 || n_kv > 4096)
        return fail(NOBLE_ERR_INVALID_ARG, "n_q=%lld, n_kv=%lld not in 1..4096", (long long)n_q, (long long)n_kv);
    return NOBLE_OK;
}
noble_status check_dtype(int32_t dtype)
{
    if (dtype != NOBLE_BF16 && dtype != NOBLE_FP32) return fail(NOBLE_ERR_UNSUPPORTED, "dtype %d not supported", (int)dtype);
    return NOBLE_OK;
}
size_t esize(int32_t dtype) { return dtype == NOBLE_BF16 ? 2 : 4; }

noble_status check_heads(const noble_heads *x, const char *name, int64_t T, int64_t n, int64_t d, int32_t dtype, bool written)
{
    if (!x) return fail(NOBLE_ERR_INVALID_ARG, "%s is NULL", name);
    NOBLE_TRY(check_ptr(x->p, name, T == 0));
    const int64_t unit = 16 / (int64_t)esize(dtype);
    if (x->row % unit || x->head % unit)
        return fail(NOBLE_ERR_MISALIGNED, "%s: strides %lld, %lld are not multiples of 16 bytes", name, (long long)x->row,
                    (long long)x->head);
    const int64_t most = int64_t(1) << 44;
    if (x->row > most || x->row < -most || x->head > most || x->head < -most)
        return fail(NOBLE_ERR_UNSUPPORTED, "%s: strides %lld, %lld too large", name, (long long)x->row, (long long)x->head);
    if (written) {
        const int64_t row = T > 1 ? std::llabs(x->row) : INT64_MAX, head = n > 1 ? std::llabs(x->head) : INT64_MAX;
        const bool token_major = n == 1 ? row >= d : head >= d && (T <= 1 || row >= (n - 1) * head + d);
        const bool head_major = T <= 1 ? head >= d : row >= d && (n == 1 || head >= (T - 1) * row + d);
        if (!token_major && !head_major)
            return fail(NOBLE_ERR_UNSUPPORTED, "%s: elements overlap (strides %lld, %lld)", name, (long long)x->row,
                        (long long)x->head);
    }
    return NOBLE_OK;
}

template <typename T>
attn::Heads<T> heads(const noble_heads *x)
{
    if (!x) return {nullptr, 0, 0};
    return {static_cast<T *>(x->p), x->row, x->head};
}

// Dynamic shared memory beyond 48 KB has to be allowed for each kernel, in each context; a
// kernel asks for the same number of bytes every time.
template <auto KERN>
noble_status allow(size_t bytes)
{
    static std::atomic<CUcontext> done{nullptr};
    const CUcontext ctx = current_context();
    if (ctx && done.load(std::memory_order_relaxed) == ctx) return NOBLE_OK;
    if (cudaFuncSetAttribute(KERN, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess)
        return fail(NOBLE_ERR_CUDA, "shared memory of %zu bytes: %s", bytes, cudaGetErrorString(cudaGetLastError()));
    done.store(current_context(), std::memory_order_relaxed);
    return NOBLE_OK;
}

// ---------------------------------------------------------------- rotary positions
noble_status validate(const noble_rope_desc *d)
{
    if (!d) return fail(NOBLE_ERR_INVALID_ARG, "desc is NULL");
    if (d->T < 0 || d->positions < 0 || !(d->eps >= 0.f) || !std::isfinite(d->eps))
        return fail(NOBLE_ERR_INVALID_ARG, "T=%lld, positions=%lld, eps=%g", (long long)d->T, (long long)d->positions, d->eps);
    NOBLE_TRY(heads_count(d->n_q, d->n_kv));
    if (d->T > INT32_MAX || d->positions > INT32_MAX) return fail(NOBLE_ERR_UNSUPPORTED, "T and positions go up to 2^31-1");
    if (d->d < 8 || d->d > 256 || d->d % 8) return fail(NOBLE_ERR_UNSUPPORTED, "d=%lld is not a multiple of 8 from 8 to 256", (long long)d->d);
    if (d->rot < 0 || d->rot > d->d || d->rot % 2)
        return fail(NOBLE_ERR_UNSUPPORTED, "rot=%lld is not even and from 0 to d", (long long)d->rot);
    NOBLE_TRY(check_dtype(d->dtype));
    if (d->flags & ~(NOBLE_ROPE_INTERLEAVED | NOBLE_ROPE_NORM)) return fail(NOBLE_ERR_UNSUPPORTED, "unknown flags 0x%x", d->flags);
    return NOBLE_OK;
}

int rope_mode(const noble_rope_desc *d)
{
    if (d->rot == 0) return rope::kHalf;
    if (d->flags & NOBLE_ROPE_INTERLEAVED) return d->rot % 8 == 0 ? rope::kInterleaved : rope::kAny;
    return d->rot % 16 == 0 ? rope::kHalf : rope::kAny;
}
int lanes_per_head(int64_t d)
{
    int lp = 1;
    while (lp * 8 < d) lp *= 2;
    return lp;
}
int64_t rope_batches(int64_t heads, int64_t d) { return ceil_div(heads, rope::kPasses * (32 / lanes_per_head(d))); }
// blocks of the backward: they set how many partial sums there are
int64_t rope_bwd_blocks(const noble_rope_desc *d)
{
    const int64_t per = std::max(rope_batches(d->n_q, d->d), rope_batches(d->n_kv, d->d));
    return std::max<int64_t>(1, std::min<int64_t>(ceil_div(d->T * per, rope::kWarps), (d->dtype == NOBLE_BF16 ? rope::kBwdBlocks<bf> : rope::kBwdBlocks<float>)*kSms));
}

template <typename T>
rope::Args<T> rope_args(const noble_rope_desc *d, const noble_heads *q, const noble_heads *k, const int32_t *pos,
                        const float *table, const float *gain_q, const float *gain_k)
{
    rope::Args<T> a{};
    a.q = heads<const T>(q), a.k = heads<const T>(k);
    a.pos = pos, a.table = table;
    a.norm = (d->flags & NOBLE_ROPE_NORM) != 0;
    a.interleaved = (d->flags & NOBLE_ROPE_INTERLEAVED) != 0;
    a.gain_q = a.norm ? gain_q : nullptr, a.gain_k = a.norm ? gain_k : nullptr;
    a.tokens = d->T, a.n_q = (int)d->n_q, a.n_kv = (int)d->n_kv, a.d = (int)d->d, a.rot = (int)d->rot;
    // eps 0: places without a head hold zeros, which times a finite factor stay 0; no head whose
    // norm fp32 can hold notices
    a.positions = (int)d->positions, a.eps = std::max(d->eps, std::numeric_limits<float>::denorm_min());
    a.lp = lanes_per_head(d->d), a.inv_d = 1.f / (float)d->d;
    a.batches_q = (int)rope_batches(d->n_q, d->d), a.batches_kv = (int)rope_batches(d->n_kv, d->d);
    return a;
}

// f(mode, lanes per head) as constants; heads of 64 and 128 features have kernels of their own
template <class F>
void rope_kernel(int mode, int lp, F &&f)
{
    auto with = [&](auto m) {
        if (lp == 8) f(m, std::integral_constant<int, 8>{});
        else if (lp == 16) f(m, std::integral_constant<int, 16>{});
        else f(m, std::integral_constant<int, 0>{});
    };
    if (mode == rope::kHalf) with(std::integral_constant<int, rope::kHalf>{});
    else if (mode == rope::kInterleaved) with(std::integral_constant<int, rope::kInterleaved>{});
    else f(std::integral_constant<int, rope::kAny>{}, std::integral_constant<int, 0>{});
}

template <bool APPEND, typename T>
noble_status rope_fwd_launch(const noble_rope_desc *d, rope::Args<T> &a, cudaStream_t st)
{
    a.status = status_ptr();
    if (!a.status) return fail(NOBLE_ERR_CUDA, "status word address");
    // one batch a warp while that leaves SMs idle, else all batches of a token, which then
    // share its cosines and sines.  Forward, 16 + 16 heads, us one a warp and all, at 15 (heads of
    // 64: 13), 26 and 52 batches per SM: heads of 128 bf16 4.0 and 6.3, 7.0 and 6.3, 9.8 and 8.4; fp32
    // 6.1 and 10.4, 10.4 and 10.5, 18.7 and 16.2; of 64 bf16 3.6 and 4.1, 6.7 and 5.6, 9.1 and 9.6;
    // fp32 5.9 and 6.4, 10.2 and 9.3, 18.3 and 17.2
    const int all = a.batches_q + (APPEND ? 2 : 1) * a.batches_kv;
    a.take = a.tokens * all <= 24 * kSms ? 1 : all;
    a.groups = (int)ceil_div(all, a.take);
    const int64_t blocks = ceil_div(a.tokens * a.groups, rope::kWarps);
    if (blocks > INT32_MAX) return fail(NOBLE_ERR_UNSUPPORTED, "%lld tokens of so many heads", (long long)a.tokens);
    const KernelInfo ki{APPEND ? "kv_append" : "rope_fwd", kBoundHbm, 0.0,
                        2.0 * sizeof(T) * a.tokens * a.d * (a.n_q + (APPEND ? 2 : 1) * a.n_kv)};
    const int mode = rope_mode(d);
    noble_status allowed = NOBLE_OK;
    rope_kernel(mode, a.lp, [&](auto m, auto lp) { allowed = allow<&rope::fwd_kernel<m.value, APPEND, lp.value, T>>(rope::kFwdBytes<T>); });
    NOBLE_TRY(allowed);
    return run(st, ki, [&] {
        const dim3 grid((unsigned)blocks), block(32 * rope::kWarps);
        rope_kernel(mode, a.lp, [&](auto m, auto lp) {
            rope::fwd_kernel<m.value, APPEND, lp.value, T><<<grid, block, rope::kFwdBytes<T>, st>>>(a);
        });
    });
}

// The arguments that the three rotary entry points share.
noble_status check_rope(const noble_rope_desc *d, const int32_t *pos, const float *table, const float *gain_q,
                        const float *gain_k)
{
    NOBLE_TRY(check_ptr(pos, "pos", d->T == 0));
    NOBLE_TRY(check_ptr(table, "table", d->T == 0 || d->rot == 0 || d->positions == 0));
    NOBLE_TRY(check_ptr(gain_q, "gain_q", true));
    return check_ptr(gain_k, "gain_k", true);
}

template <typename T>
noble_status rope_bwd_launch(const noble_rope_desc *d, rope::Args<T> &a, float *dgain_q, float *dgain_k, cudaStream_t st)
{
    a.status = status_ptr();
    if (!a.status) return fail(NOBLE_ERR_CUDA, "status word address");
    const int blocks = (int)rope_bwd_blocks(d);
    const KernelInfo ki{"rope_bwd", kBoundHbm, 0.0, (a.norm ? 3.0 : 2.0) * sizeof(T) * a.tokens * a.d * (a.n_q + a.n_kv)};
    const int mode = rope_mode(d);
    noble_status allowed = NOBLE_OK;
    rope_kernel(mode, a.lp, [&](auto m, auto lp) { allowed = allow<&rope::bwd_kernel<m.value, lp.value, T>>(rope::kRingBytes<T>); });
    NOBLE_TRY(allowed);
    NOBLE_TRY(run(st, ki, [&] {
        rope_kernel(mode, a.lp, [&](auto m, auto lp) {
            rope::bwd_kernel<m.value, lp.value, T><<<blocks, 32 * rope::kWarps, rope::kRingBytes<T>, st>>>(a);
        });
    }));
    if (!a.part) return NOBLE_OK;
    const KernelInfo kg{"rope_gain", kBoundHbm, 0.0, 8.0 * blocks * a.d};
    return run(st, kg, [&] {
        rope::gain_kernel<<<(unsigned)ceil_div(2 * a.d, 8), 256, 0, st>>>(a.part, blocks, a.d, dgain_q, dgain_k);
    });
}

// ---------------------------------------------------------------- attention over documents
noble_status check_score(float scale, float softcap, int64_t window)
{
    if (!std::isfinite(scale) || !(softcap >= 0.f) || !std::isfinite(softcap) || window < 0)
        return fail(NOBLE_ERR_INVALID_ARG, "scale=%g, softcap=%g, window=%lld", scale, softcap, (long long)window);
    return NOBLE_OK;
}
noble_status check_attn_heads(int64_t n_q, int64_t n_kv, int64_t d)
{
    NOBLE_TRY(heads_count(n_q, n_kv));
    if (n_q % n_kv) return fail(NOBLE_ERR_INVALID_ARG, "n_q=%lld is not a multiple of n_kv=%lld", (long long)n_q, (long long)n_kv);
    if (d < 8 || d > 128 || d % 8) return fail(NOBLE_ERR_UNSUPPORTED, "d=%lld is not a multiple of 8 from 8 to 128", (long long)d);
    return NOBLE_OK;
}
noble_status validate(const noble_attn_desc *d)
{
    if (!d) return fail(NOBLE_ERR_INVALID_ARG, "desc is NULL");
    if (d->T < 0 || d->n_docs < 0) return fail(NOBLE_ERR_INVALID_ARG, "T=%lld, n_docs=%lld", (long long)d->T, (long long)d->n_docs);
    if (d->T > (1 << 24) || d->n_docs > (1 << 24)) return fail(NOBLE_ERR_UNSUPPORTED, "T and n_docs go up to 2^24");
    NOBLE_TRY(check_attn_heads(d->n_q, d->n_kv, d->d));
    NOBLE_TRY(check_score(d->scale, d->softcap, d->window));
    NOBLE_TRY(check_dtype(d->dtype));
    if (d->flags & ~(NOBLE_ATTN_CAUSAL | NOBLE_ATTN_SIMT_ONLY)) return fail(NOBLE_ERR_UNSUPPORTED, "unknown flags 0x%x", d->flags);
    return NOBLE_OK;
}
noble_status check_aligned4(const void *p, const char *name, bool nullable)
{
    if (!p) return nullable ? NOBLE_OK : fail(NOBLE_ERR_INVALID_ARG, "%s is NULL", name);
    if (reinterpret_cast<uintptr_t>(p) % 4) return fail(NOBLE_ERR_MISALIGNED, "%s is not 4-byte aligned", name);
    return NOBLE_OK;
}

// Parts that the query heads of a key head are split into for dk and dv: a block of 128 keys
// and all of them is one piece of work, and the longest of a causal mask is as long as an
// SM's share of all once there are two pieces per SM.  Up to four per SM, which bounds what the
// parts take (4096 tokens, 16 heads on 4 of 128 features, causal: the backward 270 us in one
// part, 203 in four; 7001 tokens, 11 documents with prefixes, capped scores: 429 and, in two,
// 377).
int attn_splits(const noble_attn_desc *d)
{
    const int64_t group = d->n_q / d->n_kv, pieces = ceil_div(d->T, attn::tc::kRows) * d->n_kv;
    if (d->dtype != NOBLE_BF16 || (d->flags & NOBLE_ATTN_SIMT_ONLY)) return 1;
    int64_t s = 1;
    for (int64_t t = 2; t <= group && pieces * s < 2 * kSms && pieces * t <= 4 * kSms; ++t)
        if (group % t == 0) s = t;
    return (int)s;
}
struct AttnWork {
    size_t delta, rest, total;  // rest: ranges of the CUDA cores, parts of the tensor cores
};
AttnWork attn_work(const noble_attn_desc *d)
{
    AttnWork w{};
    w.rest = align_up((size_t)d->T * (size_t)d->n_q * 4, 256);
    const size_t splits = (size_t)attn_splits(d), unit = 2 * attn::tc::kRows * (d->d <= 64 ? 64 : 128) * 4;
    const size_t parts = splits > 1 ? splits * (size_t)d->n_kv * (size_t)ceil_div(d->T, attn::tc::kRows) * unit : 0;
    w.total = std::max<size_t>(256, w.rest + std::max(align_up((size_t)d->T * 8, 256), parts));
    return w;
}

template <typename T>
attn::RowArgs<T> attn_args(const noble_attn_desc *d, const noble_heads *q, const noble_heads *k, const noble_heads *v,
                           const int32_t *doc_start, const int32_t *prefix, const float *slope)
{
    attn::RowArgs<T> a{};
    a.mask = {doc_start, prefix, (int)d->n_docs, (int)d->T, (int)std::min<int64_t>(d->window, 1 << 30),
              (d->flags & NOBLE_ATTN_CAUSAL) != 0};
    a.score = {d->scale, d->softcap, slope};
    a.q = heads<const T>(q), a.k = heads<const T>(k), a.v = heads<const T>(v);
    a.n_q = (int)d->n_q, a.n_kv = (int)d->n_kv, a.d = (int)d->d;
    return a;
}

template <int DP, typename T>
noble_status attn_fwd_simt(const attn::RowArgs<T> &a, cudaStream_t st)
{
    namespace s = attn::simt;
    constexpr size_t smem = s::kFwdFloats<DP> * 4;
    NOBLE_TRY((allow<&s::fwd_kernel<DP, T>>(smem)));
    const dim3 grid((unsigned)ceil_div(a.mask.T, s::kM), (unsigned)a.n_q);
    return run(st, {"attn_fwd_simt", kBoundAlu, 0.0, 0.0}, [&] { s::fwd_kernel<DP, T><<<grid, s::kThreads, smem, st>>>(a); });
}

template <typename T>
noble_status attn_prep(const attn::RowArgs<T> &a, float *delta, int2 *ranges, cudaStream_t st)
{
    namespace s = attn::simt;
    const bool wide = a.d > 64;
    const int64_t per = wide ? 16 : 32;  // heads of a block at a time
    const int64_t blocks = std::min<int64_t>(ceil_div((int64_t)a.mask.T * a.n_q, 4 * per), 4 * kSms);
    const int step_t = (int)(blocks * per / a.n_q), step_h = (int)(blocks * per % a.n_q);
    return run(st, {"attn_delta", kBoundHbm, 0.0, 2.0 * sizeof(T) * a.mask.T * a.n_q * a.d}, [&] {
        if (wide) s::delta_kernel<T, 16><<<(unsigned)blocks, 256, 0, st>>>(a, delta, ranges, step_t, step_h);
        else s::delta_kernel<T, 8><<<(unsigned)blocks, 256, 0, st>>>(a, delta, ranges, step_t, step_h);
    });
}
template <int DP, typename T>
noble_status attn_bwd_simt(const attn::RowArgs<T> &a, float *delta, const int2 *ranges, cudaStream_t st)
{
    namespace s = attn::simt;
    constexpr size_t smem = s::kBwdFloats<DP> * 4;
    NOBLE_TRY((allow<&s::dkv_kernel<DP, T>>(smem)));
    NOBLE_TRY((allow<&s::dq_kernel<DP, T>>(smem)));
    const unsigned blocks = (unsigned)ceil_div(a.mask.T, s::kM);
    NOBLE_TRY(run(st, {"attn_dq_simt", kBoundAlu, 0.0, 0.0},
                  [&] { s::dq_kernel<DP, T><<<dim3(blocks, (unsigned)a.n_q), s::kThreads, smem, st>>>(a, delta); }));
    return run(st, {"attn_dkv_simt", kBoundAlu, 0.0, 0.0},
               [&] { s::dkv_kernel<DP, T><<<dim3(blocks, (unsigned)a.n_kv), s::kThreads, smem, st>>>(a, ranges); });
}

// TMA map of a bf16 tensor of heads: dimensions (inner first) features, head, token; boxes
// of 64 features by 128 tokens of one head, 128-byte swizzle, zeros out of bounds.
bool tma_strides(const noble_heads *x, int64_t T, int64_t n)
{
    const int64_t most = int64_t(1) << 38;
    return (n == 1 || (x->head > 0 && x->head < most)) && (T == 1 || (x->row > 0 && x->row < most));
}
noble_status make_heads_map(CUtensorMap *m, const noble_heads *x, int64_t T, int64_t n, int64_t d)
{
    EncodeTiledFn enc = encode_fn();
    if (!enc) return fail(NOBLE_ERR_CUDA, "cuTensorMapEncodeTiled is unavailable");
    // a stride that nothing is reached by may have any value
    const cuuint64_t head = (cuuint64_t)(n == 1 ? d : x->head) * 2, row = (cuuint64_t)(T == 1 ? n * d : x->row) * 2;
    cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)n, (cuuint64_t)T};
    cuuint64_t strides[2] = {head, row};
    cuuint32_t box[3] = {64, 1, attn::tc::kRows};
    cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, x->p, dims, strides, box, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS)
        return fail(NOBLE_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d): %lld tokens, %lld heads of %lld", (int)r, (long long)T,
                    (long long)n, (long long)d);
    return NOBLE_OK;
}

// Score functions beyond a positive scale take the kernels' general form.
bool general_scores(const attn::Score &s) { return s.softcap > 0.f || s.slope || !(s.scale > 0.f); }

// The register split of a kernel's warpgroups draws on what it was launched with.
template <auto KERN>
bool registers_at_least(int n)
{
    static const bool ok = [n] {
        cudaFuncAttributes a{};
        return cudaFuncGetAttributes(&a, KERN) == cudaSuccess && a.numRegs >= n;
    }();
    return ok;
}

template <int DP, bool GENERAL>
noble_status attn_fwd_tc(const attn::RowArgs<bf> &a, const CUtensorMap (&maps)[3], cudaStream_t st)
{
    namespace t = attn::tc;
    using F = t::Fwd<DP>;
    constexpr auto kern = &t::fwd_kernel<DP, GENERAL>;
    if (!registers_at_least<kern>(168)) return fail(NOBLE_ERR_CUDA, "attn_fwd: registers");
    NOBLE_TRY((allow<kern>(F::kDynamic)));
    t::FwdArgs f{a, (int)ceil_div(a.mask.T, 256), status_ptr()};
    if (!f.status) return fail(NOBLE_ERR_CUDA, "status word address");
    if ((int64_t)f.tiles * a.n_q > INT32_MAX) return fail(NOBLE_ERR_UNSUPPORTED, "%d tokens of %d heads", a.mask.T, a.n_q);
    return run(st, {"attn_fwd", kBoundTensor, 0.0, 0.0},
               [&] { kern<<<f.tiles * a.n_q, F::kThreads, F::kDynamic, st>>>(maps[0], maps[1], maps[2], f); });
}
noble_status attn_fwd_tc(const noble_attn_desc *d, const attn::RowArgs<bf> &a, const noble_heads *q, const noble_heads *k,
                         const noble_heads *v, cudaStream_t st)
{
    CUtensorMap maps[3];
    NOBLE_TRY(make_heads_map(&maps[0], q, d->T, d->n_q, d->d));
    NOBLE_TRY(make_heads_map(&maps[1], k, d->T, d->n_kv, d->d));
    NOBLE_TRY(make_heads_map(&maps[2], v, d->T, d->n_kv, d->d));
    if (general_scores(a.score)) return d->d <= 64 ? attn_fwd_tc<64, true>(a, maps, st) : attn_fwd_tc<128, true>(a, maps, st);
    return d->d <= 64 ? attn_fwd_tc<64, false>(a, maps, st) : attn_fwd_tc<128, false>(a, maps, st);
}
// bf16 runs on the tensor cores unless asked otherwise or a stride is none that TMA takes.
bool attn_use_tc(const noble_attn_desc *d, std::initializer_list<std::pair<const noble_heads *, int64_t>> xs)
{
    bool ok = d->dtype == NOBLE_BF16 && !(d->flags & NOBLE_ATTN_SIMT_ONLY);
    for (auto &x : xs) ok = ok && tma_strides(x.first, d->T, x.second);
    return ok;
}

template <int DP, bool GENERAL>
noble_status attn_bwd_tc(const attn::RowArgs<bf> &a, const CUtensorMap (&maps)[4], float *delta, int splits, float *part,
                         cudaStream_t st)
{
    namespace t = attn::tc;
    using Q = t::BwdQ<DP>;
    using KV = t::BwdKV<DP>;
    constexpr auto dq = &t::dq_kernel<DP, GENERAL>, dkv = &t::dkv_kernel<DP, GENERAL>;
    if (!registers_at_least<dq>(168) || !registers_at_least<dkv>(168)) return fail(NOBLE_ERR_CUDA, "attn_bwd: registers");
    NOBLE_TRY((allow<dq>(Q::kBytes)));
    NOBLE_TRY((allow<dkv>(KV::kBytes)));
    t::BwdArgs f{a, delta, (int)ceil_div(a.mask.T, t::kRows), splits, a.n_q / (a.n_kv * splits), a.n_kv * splits, part, status_ptr()};
    if (!f.status) return fail(NOBLE_ERR_CUDA, "status word address");
    if ((int64_t)f.tiles * a.n_q > INT32_MAX) return fail(NOBLE_ERR_UNSUPPORTED, "%d tokens of %d heads", a.mask.T, a.n_q);
    NOBLE_TRY(run(st, {"attn_dq", kBoundTensor, 0.0, 0.0},
                  [&] { dq<<<f.tiles * a.n_q, Q::kThreads, Q::kBytes, st>>>(maps[0], maps[1], maps[2], maps[3], f); }));
    NOBLE_TRY(run(st, {"attn_dkv", kBoundTensor, 0.0, 0.0},
                  [&] { dkv<<<f.tiles * f.parts, KV::kThreads, KV::kBytes, st>>>(maps[0], maps[1], maps[2], maps[3], f); }));
    if (splits == 1) return NOBLE_OK;
    const KernelInfo ki{"attn_dkv_join", kBoundHbm, 0.0, 2.0 * 4 * splits * a.mask.T * a.n_kv * a.d};
    return run(st, ki, [&] { t::join_kernel<DP><<<2 * f.tiles * a.n_kv, t::kRows * DP / 32, 0, st>>>(f); });
}
template <typename T>
noble_status attn_fwd(const attn::RowArgs<T> &a, cudaStream_t st)
{
    return a.d <= 64 ? attn_fwd_simt<64, T>(a, st) : attn_fwd_simt<128, T>(a, st);
}
template <typename T>
noble_status attn_bwd(const attn::RowArgs<T> &a, float *delta, int2 *ranges, cudaStream_t st)
{
    NOBLE_TRY(attn_prep<T>(a, delta, ranges, st));
    return a.d <= 64 ? attn_bwd_simt<64, T>(a, delta, ranges, st) : attn_bwd_simt<128, T>(a, delta, ranges, st);
}

noble_status attn_bwd_tc(const noble_attn_desc *d, const attn::RowArgs<bf> &a, const noble_heads *q, const noble_heads *d_o,
                         const noble_heads *k, const noble_heads *v, float *delta, float *part, cudaStream_t st)
{
    const int splits = attn_splits(d);
    CUtensorMap maps[4];
    NOBLE_TRY(make_heads_map(&maps[0], q, d->T, d->n_q, d->d));
    NOBLE_TRY(make_heads_map(&maps[1], d_o, d->T, d->n_q, d->d));
    NOBLE_TRY(make_heads_map(&maps[2], k, d->T, d->n_kv, d->d));
    NOBLE_TRY(make_heads_map(&maps[3], v, d->T, d->n_kv, d->d));
    NOBLE_TRY(attn_prep<bf>(a, delta, nullptr, st));
    if (general_scores(a.score))
        return d->d <= 64 ? attn_bwd_tc<64, true>(a, maps, delta, splits, part, st) : attn_bwd_tc<128, true>(a, maps, delta, splits, part, st);
    return d->d <= 64 ? attn_bwd_tc<64, false>(a, maps, delta, splits, part, st) : attn_bwd_tc<128, false>(a, maps, delta, splits, part, st);
}

// ---------------------------------------------------------------- attention over the cache
noble_status validate(const noble_paged_desc *d)
{
    if (!d) return fail(NOBLE_ERR_INVALID_ARG, "desc is NULL");
    if (d->n_seq < 0 || d->q_len < 1 || d->max_pages < 0 || d->max_len < 0)
        return fail(NOBLE_ERR_INVALID_ARG, "n_seq=%lld, q_len=%lld, max_pages=%lld, max_len=%lld", (long long)d->n_seq,
                    (long long)d->q_len, (long long)d->max_pages, (long long)d->max_len);
    if (d->n_seq > 65535 || d->q_len > 64 || d->max_pages > INT32_MAX || d->max_len > INT32_MAX)
        return fail(NOBLE_ERR_UNSUPPORTED, "n_seq goes up to 65535, q_len to 64, max_pages and max_len to 2^31-1");
    NOBLE_TRY(check_attn_heads(d->n_q, d->n_kv, d->d));
    NOBLE_TRY(check_score(d->scale, d->softcap, d->window));
    NOBLE_TRY(check_dtype(d->dtype));
    if (d->flags) return fail(NOBLE_ERR_UNSUPPORTED, "unknown flags 0x%x", d->flags);
    return NOBLE_OK;
}
noble_status check_cache(const noble_kv_cache *c, int64_t n_kv, int64_t d, int32_t dtype, bool written)
{
    if (!c) return fail(NOBLE_ERR_INVALID_ARG, "cache is NULL");
    if (c->pages < 0 || c->page_size < 1) return fail(NOBLE_ERR_INVALID_ARG, "cache: pages=%lld, page_size=%lld", (long long)c->pages, (long long)c->page_size);
    if (c->pages > INT32_MAX || c->page_size > (1 << 20)) return fail(NOBLE_ERR_UNSUPPORTED, "cache: pages up to 2^31-1 of up to 2^20 tokens");
    NOBLE_TRY(check_ptr(c->k, "cache k", c->pages == 0));
    NOBLE_TRY(check_ptr(c->v, "cache v", c->pages == 0));
    const int64_t unit = 16 / (int64_t)esize(dtype), most = int64_t(1) << 31;
    if (c->page % unit || c->row % unit || c->head % unit) return fail(NOBLE_ERR_MISALIGNED, "cache: strides are not multiples of 16 bytes");
    if (c->page < 0 || c->row < 0 || c->head < 0 || c->page > most * 16 || c->row > most || c->head > most * 16)
        return fail(NOBLE_ERR_UNSUPPORTED, "cache: strides %lld, %lld, %lld", (long long)c->page, (long long)c->row, (long long)c->head);
    if (written) {
        const noble_heads one = {c->k, c->row, c->head};
        NOBLE_TRY(check_heads(&one, "cache page", c->page_size, n_kv, d, dtype, true));
        // pages one behind the other, or as the innermost but the features of a wider row
        if (c->pages > 1 && c->page < (c->page_size - 1) * c->row + (n_kv - 1) * c->head + d)
            return fail(NOBLE_ERR_UNSUPPORTED, "cache: pages overlap (stride %lld)", (long long)c->page);
    }
    return NOBLE_OK;
}

// Keys of a chunk, and chunks of the longest sequence.  `one` is the chunk with which the
// blocks of sequences of that length fill the chip once.  One sequence, or shorter chunks
// than 1024 keys: that.  Several may differ in length, and more and smaller pieces
// balance, down to an eighth of it or 1024 keys, beside which a block's start and
// the joining count.  us with chunks of 512 / 1024 / 2048 / 3456 keys: 64 sequences up to
// 32768 tokens 450 / 394 / 366 / 365 (one: 728); 16 up to 4096 39 / 35 / 53 / 79; one
// of 131072 82 / 68 / 61 / 79 (one = 1728: 58).
struct Split {
    int chunk, chunks;
};
int64_t paged_max_len(const noble_paged_desc *d) { return std::min<int64_t>(d->max_len, attn::paged::kMaxLen); }
Split paged_split(const noble_paged_desc *d)
{
    const int64_t max_len = paged_max_len(d);
    const int64_t rows = d->n_q / d->n_kv * d->q_len;
    const int64_t units = d->n_seq * d->n_kv * ceil_div(rows, attn::paged::kRows);
    const int64_t slots = kSms * (d->d <= 64 ? attn::paged::kBlocksPerSm<64> : attn::paged::kBlocksPerSm<128>);
    const int64_t one = ceil_div(max_len * std::max<int64_t>(units, 1), slots);
    // fp32 is not bound by reading: eight blocks per SM, which balances (24 sequences up to 1000
    // tokens, 16 heads of 64, with 4, 6, 8, 12 and 16 per SM: 106, 83, 73, 72 and 73 us; 16 up to
    // 8000: 644, 524, 429, 492 and 422; 32 heads on 4 of 128: 314, 220, 224, 261 and 220)
    int64_t chunk = d->dtype == NOBLE_FP32 ? ceil_div(max_len * std::max<int64_t>(units, 1), 8 * kSms)
                    : d->n_seq <= 1        ? one
                                           : std::max(one / 8, std::min<int64_t>(one, 1024));
    chunk = std::max<int64_t>(chunk, 256);
    const int64_t chunks = std::max<int64_t>(1, ceil_div(max_len, chunk));
    chunk = std::max<int64_t>(1, ceil_div(ceil_div(max_len, chunks), attn::paged::kKeys)) * attn::paged::kKeys;
    return {(int)chunk, (int)std::max<int64_t>(1, ceil_div(max_len, chunk))};
}
struct PagedWork {
    size_t ml, total;
};
PagedWork paged_work(const noble_paged_desc *d)
{
    const size_t n = (size_t)d->n_seq * d->q_len * d->n_q * paged_split(d).chunks;
    PagedWork w{};
    w.ml = align_up(n * d->d * 4, 256);
    w.total = paged_split(d).chunks > 1 ? w.ml + align_up(n * 8, 256) : 256;
    return w;
}

template <int DP, typename T>
noble_status paged_launch(const attn::paged::Args<T> &a, cudaStream_t st)
{
    namespace p = attn::paged;
    constexpr size_t smem = ((p::kRows + p::kKeys) * attn::simt::kLd<DP> + p::kRows * attn::simt::kPP) * 4;
    const int64_t rows = (int64_t)(a.n_q / a.n_kv) * a.q_len;
    const dim3 grid((unsigned)(a.chunks * ceil_div(rows, p::kRows)), (unsigned)a.n_kv, (unsigned)a.n_seq);
    if constexpr (std::is_same_v<T, bf>) {
        NOBLE_TRY(run(st, {"attn_paged", kBoundHbm, 0.0, 0.0}, [&] {
            if (a.page_size % 16 == 0) p::mma_kernel<DP, true><<<grid, p::kThreads, 0, st>>>(a);
            else p::mma_kernel<DP, false><<<grid, p::kThreads, 0, st>>>(a);
        }));
    } else {
        NOBLE_TRY((allow<&p::simt_kernel<DP, T>>(smem)));
        NOBLE_TRY(run(st, {"attn_paged_simt", kBoundHbm, 0.0, 0.0},
                      [&] { p::simt_kernel<DP, T><<<grid, p::kThreads, smem, st>>>(a); }));
    }
    if (a.chunks == 1) return NOBLE_OK;
    // warps per row: about eight chunks each
    int per_row = 1;
    while (per_row < 8 && a.chunks > 8 * per_row) per_row *= 2;
    const unsigned blocks = (unsigned)ceil_div((int64_t)a.n_seq * a.q_len * a.n_q, 8 / per_row);
    const bool pdl = pdl_ok();
    return run(st, {"attn_paged_join", kBoundHbm, 0.0, 0.0},
               [&] { launch_maybe_pdl(p::join_kernel<T>, dim3(blocks), dim3(256), 0, st, pdl, a, per_row); });
}

template <typename T>
noble_status paged(const noble_paged_desc *d, const noble_heads *q, const noble_kv_cache *c, const int32_t *page_table,
                   const int32_t *kv_len, const float *slope, const noble_heads *o, float *lse, char *ws, cudaStream_t st)
{
    attn::paged::Args<T> a{};
    a.q = heads<const T>(q), a.o = heads<T>(o);
    a.k = static_cast<const T *>(c->k), a.v = static_cast<const T *>(c->v);
    a.page_table = page_table, a.kv_len = kv_len, a.lse = lse;
    a.part_o = reinterpret_cast<float *>(ws), a.part_ml = reinterpret_cast<float *>(ws + paged_work(d).ml);
    a.page = c->page, a.row = c->row, a.head = c->head;
    a.max_pages = d->max_pages, a.max_len = paged_max_len(d);
    a.pages = (int)c->pages, a.page_size = (int)c->page_size;
    a.n_seq = (int)d->n_seq, a.q_len = (int)d->q_len, a.n_q = (int)d->n_q, a.n_kv = (int)d->n_kv, a.d = (int)d->d;
    a.window = (int)std::min<int64_t>(d->window, attn::paged::kMaxLen);  // as far as any key is from its query
    const Split s = paged_split(d);
    a.chunk = s.chunk, a.chunks = s.chunks;
    a.score = {d->scale, d->softcap, slope};
    a.status = status_ptr();
    if (!a.status) return fail(NOBLE_ERR_CUDA, "status word address");
    return a.d <= 64 ? paged_launch<64, T>(a, st) : paged_launch<128, T>(a, st);
}

}  // namespace
}  // namespace noble

using namespace noble;

extern "C" {

noble_status noble_rope_table(int64_t positions, int64_t rot, const noble_rope_scaling *scaling, float *table,
                              noble_stream stream)
{
    g_last_error[0] = 0;
    g_call_kernels = 0;
    if (positions < 0 || positions > INT32_MAX || rot < 0 || rot > 256 || rot % 2)
        return fail(NOBLE_ERR_INVALID_ARG, "positions=%lld, rot=%lld", (long long)positions, (long long)rot);
    const noble_rope_scaling plain = {10000.0, 1.0, 1.0, 0.0, 0.0, 1.0}, &s = scaling ? *scaling : plain;
    if (!(s.base > 0.0) || !std::isfinite(s.base) || !(s.factor > 0.0) || !std::isfinite(s.factor) || !(s.original > 0.0) ||
        !std::isfinite(s.original) || !(s.low_turns <= s.high_turns) || !std::isfinite(s.amplitude))
        return fail(NOBLE_ERR_INVALID_ARG, "scaling: base %g, factor %g, original %g, turns %g to %g, amplitude %g", s.base,
                    s.factor, s.original, s.low_turns, s.high_turns, s.amplitude);
    NOBLE_TRY(check_ptr(table, "table", positions * rot == 0));
    NOBLE_TRY(check_device());
    if (positions * rot == 0) return NOBLE_OK;
    const rope::TableArgs a = {std::log2(s.base), s.factor, s.original, s.low_turns, s.high_turns, s.amplitude, positions, (int)rot};
    const unsigned blocks = (unsigned)std::min<int64_t>(ceil_div(positions * rot / 2, 256), 8 * kSms);
    return run((cudaStream_t)stream, {"rope_table", kBoundAlu, 0.0, 4.0 * positions * rot},
               [&] { rope::table_kernel<<<blocks, 256, 0, (cudaStream_t)stream>>>(a, table); });
}

noble_status noble_rope_fwd(const noble_rope_desc *desc, const noble_heads *q, const noble_heads *k, const int32_t *pos,
                            const float *table, const float *gain_q, const float *gain_k, const noble_heads *q_out,
                            const noble_heads *k_out, noble_stream stream)
{
    g_last_error[0] = 0;
    g_call_kernels = 0;
    NOBLE_TRY(validate(desc));
    NOBLE_TRY(check_rope(desc, pos, table, gain_q, gain_k));
    NOBLE_TRY(check_heads(q, "q", desc->T, desc->n_q, desc->d, desc->dtype, false));
    NOBLE_TRY(check_heads(k, "k", desc->T, desc->n_kv, desc->d, desc->dtype, false));
    NOBLE_TRY(check_heads(q_out, "q_out", desc->T, desc->n_q, desc->d, desc->dtype, true));
    NOBLE_TRY(check_heads(k_out, "k_out", desc->T, desc->n_kv, desc->d, desc->dtype, true));
    NOBLE_TRY(check_device());
    if (desc->T == 0) return NOBLE_OK;
    auto go = [&](auto zero) {
        using T = decltype(zero);
        rope::Args<T> a = rope_args<T>(desc, q, k, pos, table, gain_q, gain_k);
        a.q_out = heads<T>(q_out), a.k_out = heads<T>(k_out);
        return rope_fwd_launch<false, T>(desc, a, (cudaStream_t)stream);
    };
    return desc->dtype == NOBLE_BF16 ? go(bf{}) : go(float{});
}

size_t noble_rope_bwd_workspace_bytes(const noble_rope_desc *desc)
{
    if (validate(desc) != NOBLE_OK) return 0;
    return align_up((size_t)rope_bwd_blocks(desc) * 2 * (size_t)desc->d * 4, 256);
}

noble_status noble_rope_bwd(const noble_rope_desc *desc, const noble_heads *dq, const noble_heads *dk, const noble_heads *q,
                            const noble_heads *k, const int32_t *pos, const float *table, const float *gain_q,
                            const float *gain_k, const noble_heads *dq_in, const noble_heads *dk_in, float *dgain_q,
                            float *dgain_k, void *workspace, size_t workspace_bytes, noble_stream stream)
{
    g_last_error[0] = 0;
    g_call_kernels = 0;
    NOBLE_TRY(validate(desc));
    const bool norm = (desc->flags & NOBLE_ROPE_NORM) != 0;
    NOBLE_TRY(check_rope(desc, pos, table, gain_q, gain_k));
    NOBLE_TRY(check_heads(dq, "dq", desc->T, desc->n_q, desc->d, desc->dtype, false));
    NOBLE_TRY(check_heads(dk, "dk", desc->T, desc->n_kv, desc->d, desc->dtype, false));
    if (norm) {
        NOBLE_TRY(check_heads(q, "q", desc->T, desc->n_q, desc->d, desc->dtype, false));
        NOBLE_TRY(check_heads(k, "k", desc->T, desc->n_kv, desc->d, desc->dtype, false));
    }
    NOBLE_TRY(check_heads(dq_in, "dq_in", desc->T, desc->n_q, desc->d, desc->dtype, true));
    NOBLE_TRY(check_heads(dk_in, "dk_in", desc->T, desc->n_kv, desc->d, desc->dtype, true));
    NOBLE_TRY(check_ptr(dgain_q, "dgain_q", true));
    NOBLE_TRY(check_ptr(dgain_k, "dgain_k", true));
    const bool sums = norm && (dgain_q || dgain_k);
    if (sums) {
        NOBLE_TRY(check_ptr(workspace, "workspace", false));
        if (workspace_bytes < noble_rope_bwd_workspace_bytes(desc))
            return fail(NOBLE_ERR_BUFFER_TOO_SMALL, "workspace_bytes=%zu < %zu", workspace_bytes, noble_rope_bwd_workspace_bytes(desc));
    }
    NOBLE_TRY(check_device());
    if (desc->T == 0 && !sums) return NOBLE_OK;
    auto go = [&](auto zero) {
        using T = decltype(zero);
        rope::Args<T> a = rope_args<T>(desc, norm ? q : nullptr, norm ? k : nullptr, pos, table, gain_q, gain_k);
        a.dq = heads<const T>(dq), a.dk = heads<const T>(dk);
        a.q_out = heads<T>(dq_in), a.k_out = heads<T>(dk_in);
        a.part = sums ? static_cast<float *>(workspace) : nullptr;
        return rope_bwd_launch<T>(desc, a, dgain_q, dgain_k, (cudaStream_t)stream);
    };
    return desc->dtype == NOBLE_BF16 ? go(bf{}) : go(float{});
}

noble_status noble_kv_append(const noble_rope_desc *desc, const noble_heads *q, const noble_heads *k, const noble_heads *v,
                             const int32_t *pos, const int64_t *slots, const float *table, const float *gain_q,
                             const float *gain_k, const noble_heads *q_out, const noble_kv_cache *cache, noble_stream stream)
{
    g_last_error[0] = 0;
    g_call_kernels = 0;
    NOBLE_TRY(validate(desc));
    NOBLE_TRY(check_rope(desc, pos, table, gain_q, gain_k));
    NOBLE_TRY(check_ptr(slots, "slots", desc->T == 0));
    NOBLE_TRY(check_heads(q, "q", desc->T, desc->n_q, desc->d, desc->dtype, false));
    NOBLE_TRY(check_heads(k, "k", desc->T, desc->n_kv, desc->d, desc->dtype, false));
    NOBLE_TRY(check_heads(v, "v", desc->T, desc->n_kv, desc->d, desc->dtype, false));
    NOBLE_TRY(check_heads(q_out, "q_out", desc->T, desc->n_q, desc->d, desc->dtype, true));
    NOBLE_TRY(check_cache(cache, desc->n_kv, desc->d, desc->dtype, true));
    NOBLE_TRY(check_device());
    if (desc->T == 0) return NOBLE_OK;
    auto go = [&](auto zero) {
        using T = decltype(zero);
        rope::Args<T> a = rope_args<T>(desc, q, k, pos, table, gain_q, gain_k);
        a.v = heads<const T>(v), a.q_out = heads<T>(q_out);
        a.slots = slots, a.k_cache = static_cast<T *>(cache->k), a.v_cache = static_cast<T *>(cache->v);
        a.capacity = cache->pages * cache->page_size, a.page_size = (int)cache->page_size;
        a.page = cache->page, a.row = cache->row, a.head = cache->head;
        return rope_fwd_launch<true, T>(desc, a, (cudaStream_t)stream);
    };
    return desc->dtype == NOBLE_BF16 ? go(bf{}) : go(float{});
}

noble_status noble_attn_fwd(const noble_attn_desc *desc, const noble_heads *q, const noble_heads *k, const noble_heads *v,
                            const int32_t *doc_start, const int32_t *prefix, const float *slope, const noble_heads *o,
                            float *lse, noble_stream stream)
{
    g_last_error[0] = 0;
    g_call_kernels = 0;
    NOBLE_TRY(validate(desc));
    NOBLE_TRY(check_heads(q, "q", desc->T, desc->n_q, desc->d, desc->dtype, false));
    NOBLE_TRY(check_heads(k, "k", desc->T, desc->n_kv, desc->d, desc->dtype, false));
    NOBLE_TRY(check_heads(v, "v", desc->T, desc->n_kv, desc->d, desc->dtype, false));
    NOBLE_TRY(check_aligned4(doc_start, "doc_start", desc->T == 0));
    NOBLE_TRY(check_aligned4(prefix, "prefix", true));
    NOBLE_TRY(check_aligned4(slope, "slope", true));
    NOBLE_TRY(check_heads(o, "o", desc->T, desc->n_q, desc->d, desc->dtype, true));
    NOBLE_TRY(check_ptr(lse, "lse", desc->T == 0));
    NOBLE_TRY(check_device());
    if (desc->T == 0) return NOBLE_OK;
    auto go = [&](auto zero) {
        using T = decltype(zero);
        attn::RowArgs<T> a = attn_args<T>(desc, q, k, v, doc_start, prefix, slope);
        a.out = heads<T>(o), a.lse = lse;
        if constexpr (std::is_same_v<T, bf>)
            if (attn_use_tc(desc, {{q, desc->n_q}, {k, desc->n_kv}, {v, desc->n_kv}}))
                return attn_fwd_tc(desc, a, q, k, v, (cudaStream_t)stream);
        return attn_fwd<T>(a, (cudaStream_t)stream);
    };
    return desc->dtype == NOBLE_BF16 ? go(bf{}) : go(float{});
}

size_t noble_attn_bwd_workspace_bytes(const noble_attn_desc *desc)
{
    if (validate(desc) != NOBLE_OK) return 0;
    return attn_work(desc).total;
}

noble_status noble_attn_bwd(const noble_attn_desc *desc, const noble_heads *d_o, const noble_heads *q, const noble_heads *k,
                            const noble_heads *v, const int32_t *doc_start, const int32_t *prefix, const float *slope,
                            const noble_heads *o, const float *lse, const noble_heads *dq, const noble_heads *dk,
                            const noble_heads *dv, void *workspace, size_t workspace_bytes, noble_stream stream)
{
    g_last_error[0] = 0;
    g_call_kernels = 0;
    NOBLE_TRY(validate(desc));
    const int64_t T = desc->T;
    NOBLE_TRY(check_heads(d_o, "d_o", T, desc->n_q, desc->d, desc->dtype, false));
    NOBLE_TRY(check_heads(q, "q", T, desc->n_q, desc->d, desc->dtype, false));
    NOBLE_TRY(check_heads(k, "k", T, desc->n_kv, desc->d, desc->dtype, false));
    NOBLE_TRY(check_heads(v, "v", T, desc->n_kv, desc->d, desc->dtype, false));
    NOBLE_TRY(check_aligned4(doc_start, "doc_start", T == 0));
    NOBLE_TRY(check_aligned4(prefix, "prefix", true));
    NOBLE_TRY(check_aligned4(slope, "slope", true));
    NOBLE_TRY(check_heads(o, "o", T, desc->n_q, desc->d, desc->dtype, false));
    NOBLE_TRY(check_ptr(lse, "lse", T == 0));
    NOBLE_TRY(check_heads(dq, "dq", T, desc->n_q, desc->d, desc->dtype, true));
    NOBLE_TRY(check_heads(dk, "dk", T, desc->n_kv, desc->d, desc->dtype, true));
    NOBLE_TRY(check_heads(dv, "dv", T, desc->n_kv, desc->d, desc->dtype, true));
    NOBLE_TRY(check_ptr(workspace, "workspace", T == 0));
    if (workspace_bytes < attn_work(desc).total && T > 0)
        return fail(NOBLE_ERR_BUFFER_TOO_SMALL, "workspace_bytes=%zu < %zu", workspace_bytes, attn_work(desc).total);
    NOBLE_TRY(check_device());
    if (T == 0) return NOBLE_OK;
    auto go = [&](auto zero) {
        using E = decltype(zero);
        attn::RowArgs<E> a = attn_args<E>(desc, q, k, v, doc_start, prefix, slope);
        float *delta = static_cast<float *>(workspace);
        a.o = heads<const E>(o), a.d_o = heads<const E>(d_o), a.lse = const_cast<float *>(lse), a.delta = delta;
        a.dq = heads<E>(dq), a.dk = heads<E>(dk), a.dv = heads<E>(dv);
        char *rest = static_cast<char *>(workspace) + attn_work(desc).rest;
        if constexpr (std::is_same_v<E, bf>)
            if (attn_use_tc(desc, {{q, desc->n_q}, {d_o, desc->n_q}, {k, desc->n_kv}, {v, desc->n_kv}}))
                return attn_bwd_tc(desc, a, q, d_o, k, v, delta, reinterpret_cast<float *>(rest), (cudaStream_t)stream);
        return attn_bwd<E>(a, delta, reinterpret_cast<int2 *>(rest), (cudaStream_t)stream);
    };
    return desc->dtype == NOBLE_BF16 ? go(bf{}) : go(float{});
}

size_t noble_attn_paged_workspace_bytes(const noble_paged_desc *desc)
{
    if (validate(desc) != NOBLE_OK) return 0;
    return paged_work(desc).total;
}

noble_status noble_attn_paged(const noble_paged_desc *desc, const noble_heads *q, const noble_kv_cache *cache,
                              const int32_t *page_table, const int32_t *kv_len, const float *slope, const noble_heads *o,
                              float *lse, void *workspace, size_t workspace_bytes, noble_stream stream)
{
    g_last_error[0] = 0;
    g_call_kernels = 0;
    NOBLE_TRY(validate(desc));
    const int64_t rows = desc->n_seq * desc->q_len;
    NOBLE_TRY(check_heads(q, "q", rows, desc->n_q, desc->d, desc->dtype, false));
    NOBLE_TRY(check_cache(cache, desc->n_kv, desc->d, desc->dtype, false));
    NOBLE_TRY(check_aligned4(page_table, "page_table", rows == 0 || desc->max_pages == 0));
    NOBLE_TRY(check_aligned4(kv_len, "kv_len", rows == 0));
    NOBLE_TRY(check_aligned4(slope, "slope", true));
    NOBLE_TRY(check_heads(o, "o", rows, desc->n_q, desc->d, desc->dtype, true));
    NOBLE_TRY(check_aligned4(lse, "lse", true));
    if (paged_split(desc).chunks > 1 && rows > 0) NOBLE_TRY(check_ptr(workspace, "workspace", false));
    if (workspace_bytes < paged_work(desc).total && paged_split(desc).chunks > 1 && rows > 0)
        return fail(NOBLE_ERR_BUFFER_TOO_SMALL, "workspace_bytes=%zu < %zu", workspace_bytes, paged_work(desc).total);
    NOBLE_TRY(check_device());
    if (rows == 0) return NOBLE_OK;
    cudaStream_t st = (cudaStream_t)stream;
    if (desc->dtype == NOBLE_BF16)
        return paged<bf>(desc, q, cache, page_table, kv_len, slope, o, lse, static_cast<char *>(workspace), st);
    return paged<float>(desc, q, cache, page_table, kv_len, slope, o, lse, static_cast<char *>(workspace), st);
}

noble_status noble_debug_rows_again(uint64_t *count, noble_stream stream)
{
    g_last_error[0] = 0;
    if (!count) return fail(NOBLE_ERR_INVALID_ARG, "count is NULL");
    NOBLE_TRY(check_device());
    const unsigned long long zero = 0;
    unsigned long long v = 0;
    cudaError_t e = cudaStreamSynchronize((cudaStream_t)stream);
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&v, attn::g_rows_again, sizeof(v));
    if (e == cudaSuccess && v) e = cudaMemcpyToSymbol(attn::g_rows_again, &zero, sizeof(zero));
    if (e != cudaSuccess) return fail(NOBLE_ERR_CUDA, "count: %s", cudaGetErrorString(e));
    *count = v;
    return NOBLE_OK;
}

}  // extern "C"
