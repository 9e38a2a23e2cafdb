// C-ABI entry points around the projections of a training step (declared in
// include/noble.h): layer norm, embedding, optimizer step by orthogonalised momentum.
//
// Host side only: argument checks, workspaces and kernel dispatch.
#include <algorithm>
#include <cmath>

#include "host.cuh"
#include "embed.cuh"
#include "muon.cuh"
#include "norm.cuh"

namespace noble {
namespace {

using bf = __nv_bfloat16;
constexpr int kSms = 152;  // of a GB300; rules that choose between orders of sums take this, not the device's

noble_status check_dtype(int32_t dtype)
{
    if (dtype != NOBLE_BF16 && dtype != NOBLE_FP32) return fail(NOBLE_ERR_UNSUPPORTED, "dtype %d not supported", (int)dtype);
    return NOBLE_OK;
}
noble_status check_workspace(const void *p, size_t bytes, size_t need)
{
    NOBLE_TRY(check_ptr(p, "workspace", need == 0));
    if (bytes < need) return fail(NOBLE_ERR_BUFFER_TOO_SMALL, "workspace_bytes=%zu, needs %zu", bytes, need);
    return NOBLE_OK;
}
noble_status get_status(uint32_t **p)
{
    *p = status_ptr();
    return *p ? NOBLE_OK : fail(NOBLE_ERR_CUDA, "status word address");
}

// ---------------------------------------------------------------- layer norm
noble_status validate(const noble_norm_desc *d)
{
    if (!d) return fail(NOBLE_ERR_INVALID_ARG, "desc is NULL");
    if (d->T < 0 || !(d->eps >= 0.f) || !std::isfinite(d->eps))
        return fail(NOBLE_ERR_INVALID_ARG, "T=%lld, eps=%g", (long long)d->T, d->eps);
    if (d->T > INT32_MAX) return fail(NOBLE_ERR_UNSUPPORTED, "T goes up to 2^31-1");
    if (d->d < 8 || d->d > 16384 || d->d % 8)
        return fail(NOBLE_ERR_UNSUPPORTED, "d=%lld is not a multiple of 8 from 8 to 16384", (long long)d->d);
    NOBLE_TRY(check_dtype(d->dtype));
    if (d->flags) return fail(NOBLE_ERR_UNSUPPORTED, "unknown flags 0x%x", d->flags);
    return NOBLE_OK;
}

// f(16-byte pieces of a row per thread, warps of a row)
template <class F>
void norm_split(int vecs, int most, F &&f)
{
    if (vecs <= 32 || most == 1) f(std::integral_constant<int, 1>{}, (int)ceil_div(vecs, 32));
    else if (vecs <= 64 || most == 2) f(std::integral_constant<int, 2>{}, (int)ceil_div(vecs, 64));
    else f(std::integral_constant<int, 4>{}, (int)ceil_div(vecs, 128));
}
int norm_groups(int warps) { return std::max(1, norm::kThreads / 32 / warps); }

template <typename T>
noble_status norm_fwd(const noble_norm_desc *d, const void *x, const void *res, const float *gain, const float *bias,
                      void *sum, void *y, float *stats, cudaStream_t st)
{
    norm::FwdArgs<T> a{static_cast<const T *>(x), static_cast<const T *>(res), gain, bias, static_cast<T *>(sum),
                       static_cast<T *>(y), reinterpret_cast<float2 *>(stats), d->T, (int)d->d, 0, 1.f / (float)d->d,
                       // eps 0: a row of equal elements gives 0 times a finite factor
                       std::max(d->eps, 1e-37f)};
    const KernelInfo ki{"norm_fwd", kBoundHbm, 0.0, (double)sizeof(T) * d->T * d->d * (res ? 4 : 2)};
    return run(st, ki, [&] {
        norm_split((int)(d->d / norm::Vec<T>::n), 4, [&](auto nv, int warps) {
            a.warps = warps;
            const int groups = norm_groups(warps);
            const dim3 grid((unsigned)ceil_div(d->T, groups)), block(32 * warps * groups);
            if (res) norm::fwd_kernel<T, nv.value, true><<<grid, block, 0, st>>>(a);
            else norm::fwd_kernel<T, nv.value, false><<<grid, block, 0, st>>>(a);
        });
    });
}

// Rows of a part of the sums for dgain and dbias: about two blocks per SM, and at most 512, so that
// sums of like rows stay short.
int norm_rows_per_part(const noble_norm_desc *d)
{
    return (int)std::min<int64_t>(512, std::max<int64_t>(8, ceil_div(d->T, 2 * kSms)));
}

template <typename T>
noble_status norm_bwd(const noble_norm_desc *d, const void *dy, const void *s, const float *stats, const float *gain,
                      const void *dstream, void *dx, float *dgain, float *dbias, void *workspace, cudaStream_t st)
{
    norm::BwdArgs<T> a{static_cast<const T *>(dy), static_cast<const T *>(s), static_cast<const T *>(dstream),
                       reinterpret_cast<const float2 *>(stats), gain, static_cast<T *>(dx),
                       dgain || dbias ? static_cast<float *>(workspace) : nullptr, d->T, (int)d->d, 0,
                       norm_rows_per_part(d), 1.f / (float)d->d};
    const int64_t parts = ceil_div(d->T, a.rows_per_part);
    const KernelInfo ki{"norm_bwd", kBoundHbm, 0.0, (double)sizeof(T) * d->T * d->d * (dstream ? 4 : 3)};
    NOBLE_TRY(run(st, ki, [&] {
        norm_split((int)(d->d / norm::Vec<T>::n), 16 / norm::Vec<T>::n, [&](auto nv, int warps) {
            a.warps = warps;
            const int groups = norm_groups(warps);
            const size_t smem = groups > 1 ? (size_t)groups * 2 * d->d * 4 : 0;
            const dim3 grid((unsigned)parts), block(32 * warps * groups);
            if constexpr (nv.value * norm::Vec<T>::n <= 16) {
                if (dstream) norm::bwd_kernel<T, nv.value, true><<<grid, block, smem, st>>>(a);
                else norm::bwd_kernel<T, nv.value, false><<<grid, block, smem, st>>>(a);
            }
        });
    }));
    if (!a.part) return NOBLE_OK;
    SplitJobs J{};
    for (float *out : {dgain, dbias}) {
        if (!out) continue;
        const int j = J.njobs++;
        J.part[j] = a.part + (out == dgain ? 0 : d->d);
        J.out[j] = out, J.n[j] = d->d, J.stride[j] = 2 * d->d;
        J.begin[j + 1] = J.begin[j] + d->d;
    }
    J.nparts = (int)parts;
    return run(st, {"norm_join", kBoundHbm, 0.0, 8.0 * parts * d->d},
               [&] { norm::join_kernel<<<(unsigned)ceil_div(J.begin[J.njobs], 32), 256, 0, st>>>(J); });
}

// ---------------------------------------------------------------- embedding
noble_status validate(const noble_embed_desc *d)
{
    if (!d) return fail(NOBLE_ERR_INVALID_ARG, "desc is NULL");
    if (d->T < 0 || d->vocab < 1 || !std::isfinite(d->scale))
        return fail(NOBLE_ERR_INVALID_ARG, "T=%lld, vocab=%lld, scale=%g", (long long)d->T, (long long)d->vocab, d->scale);
    if (d->T > (1 << 24) || d->vocab > (1 << 28)) return fail(NOBLE_ERR_UNSUPPORTED, "T goes up to 2^24, vocab up to 2^28");
    if (d->d < 8 || d->d > 65536 || d->d % 8)
        return fail(NOBLE_ERR_UNSUPPORTED, "d=%lld is not a multiple of 8 from 8 to 65536", (long long)d->d);
    NOBLE_TRY(check_dtype(d->dtype));
    if (d->flags) return fail(NOBLE_ERR_UNSUPPORTED, "unknown flags 0x%x", d->flags);
    return NOBLE_OK;
}

struct EmbedWork {
    size_t count, head, begin, rank, list, long_row, long_at, piece, part, total;
};
EmbedWork embed_work(const noble_embed_desc *d)
{
    EmbedWork w{};
    if (d->T <= embed::kFewTokens) {
        w.total = 256;
        return w;
    }
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t p = at;
        at = align_up(at + bytes, 256);
        return p;
    };
    // long lists have at least kShort + 1 tokens, so that there are at most T / kShort of them, and of
    // pieces
    const size_t T = (size_t)d->T, V = (size_t)d->vocab, lists = T / embed::kShort + 1;
    static_assert(embed::kPiece >= 2 * embed::kShort, "a list of n > kShort tokens has at most n / kShort pieces");
    w.head = take(16);
    w.count = take(4 * V);
    w.begin = take(4 * V);
    w.rank = take(4 * T);
    w.list = take(4 * T);
    w.long_row = take(4 * lists);
    w.long_at = take(4 * lists);
    w.piece = take(8 * lists);
    w.part = take(4 * lists * (size_t)d->d);
    w.total = at;
    return w;
}

template <typename T>
noble_status embed_fwd(const noble_embed_desc *d, const int32_t *ids, const void *table, void *y, cudaStream_t st)
{
    embed::FwdArgs<T> a{ids, static_cast<const T *>(table), static_cast<T *>(y), d->T, (int)d->vocab, (int)d->d, d->scale, nullptr};
    NOBLE_TRY(get_status(&a.status));
    const int vecs = (int)(d->d / norm::Vec<T>::n);
    return run(st, {"embed_fwd", kBoundHbm, 0.0, 2.0 * sizeof(T) * d->T * d->d}, [&] {
        const dim3 grid((unsigned)ceil_div(d->T, 8), (unsigned)std::min<int64_t>(ceil_div(vecs, 128), 64));
        embed::fwd_kernel<T, 4><<<grid, 256, 0, st>>>(a);
    });
}

template <typename T>
noble_status embed_bwd(const noble_embed_desc *d, const int32_t *ids, const void *dy, float *dtable, void *workspace, cudaStream_t st)
{
    embed::BwdArgs<T> a{};
    a.ids = ids, a.dy = static_cast<const T *>(dy), a.dtable = dtable;
    a.tokens = d->T, a.vocab = (int)d->vocab, a.d = (int)d->d, a.scale = d->scale;
    NOBLE_TRY(get_status(&a.status));
    const int vecs = (int)(d->d / norm::Vec<T>::n);
    const unsigned slices = (unsigned)ceil_div(vecs, 32);
    const double out = 4.0 * d->vocab * d->d, in = (double)sizeof(T) * d->T * d->d;
    if (d->T <= embed::kFewTokens)
        return run(st, {"embed_few", kBoundHbm, 0.0, in + out}, [&] {
            embed::few_kernel<T><<<dim3((unsigned)ceil_div(d->vocab, embed::kFewRows), slices), 256, 0, st>>>(a);
        });
    const EmbedWork w = embed_work(d);
    char *ws = static_cast<char *>(workspace);
    auto at = [&](size_t off) { return reinterpret_cast<uint32_t *>(ws + off); };
    a.head = at(w.head), a.count = at(w.count), a.begin = at(w.begin), a.rank = at(w.rank), a.list = at(w.list);
    a.long_row = at(w.long_row), a.long_at = at(w.long_at);
    a.piece = reinterpret_cast<uint2 *>(ws + w.piece), a.part = reinterpret_cast<float *>(ws + w.part);
    if (memset_async(ws, 0, w.count + 4 * (size_t)d->vocab, st) != cudaSuccess)
        return fail(NOBLE_ERR_CUDA, "memset: %s", cudaGetErrorString(cudaGetLastError()));
    const unsigned per_token = (unsigned)ceil_div(d->T, 256), per_row = (unsigned)ceil_div(d->vocab, 256);
    const KernelInfo index{"embed_index", kBoundHbm, 0.0, 0.0};
    NOBLE_TRY(run(st, index, [&] { embed::count_kernel<T><<<per_token, 256, 0, st>>>(a); }));
    NOBLE_TRY(run(st, index, [&] { embed::lists_kernel<T><<<per_row, 256, 0, st>>>(a); }));
    NOBLE_TRY(run(st, index, [&] { embed::place_kernel<T><<<per_token, 256, 0, st>>>(a); }));
    const size_t bits = (size_t)std::min<int64_t>(embed::kWindow, (int64_t)align_up((size_t)d->T, 32)) / 8;
    NOBLE_TRY(run(st, index, [&] { embed::order_kernel<T><<<4 * kSms, 256, bits, st>>>(a); }));
    NOBLE_TRY(run(st, {"embed_sum", kBoundHbm, 0.0, in + out}, [&] {
        const int64_t blocks = ceil_div(d->vocab + d->T / embed::kShort, 8);
        embed::sum_kernel<T><<<dim3((unsigned)std::min<int64_t>(blocks, 1 << 16), std::min(slices, 64u)), 256, 0, st>>>(a);
    }));
    return run(st, {"embed_join", kBoundHbm, 0.0, 0.0}, [&] {
        embed::join_kernel<T><<<dim3(kSms, (unsigned)std::min<int64_t>(ceil_div(d->d, 1024), 64)), 256, 0, st>>>(a);
    });
}

// ---------------------------------------------------------------- orthogonalised momentum
noble_status validate_muon(const noble_muon_tensor *t, int n, uint32_t flags)
{
    if (n < 0 || (n > 0 && !t)) return fail(NOBLE_ERR_INVALID_ARG, "tensors");
    if (flags & ~(NOBLE_MUON_NESTEROV | NOBLE_MUON_PRECISE)) return fail(NOBLE_ERR_UNSUPPORTED, "unknown flags 0x%x", flags);
    for (int i = 0; i < n; ++i) {
        if (t[i].rows < 0 || t[i].cols < 0 || !(t[i].lr_mult >= 0.f) || !std::isfinite(t[i].lr_mult))
            return fail(NOBLE_ERR_INVALID_ARG, "tensor %d: %lld x %lld, lr_mult %g", i, (long long)t[i].rows, (long long)t[i].cols, t[i].lr_mult);
        if (t[i].rows > 65536 || t[i].cols > 65536) return fail(NOBLE_ERR_UNSUPPORTED, "tensor %d: rows and cols go up to 65536", i);
    }
    return NOBLE_OK;
}
// Nothing that is written may be another tensor's, or its own gradient.
noble_status check_apart(const noble_muon_tensor *t, int n)
{
    for (int i = 0; i < n; ++i) {
        if (t[i].rows * t[i].cols == 0) continue;
        const void *w[4] = {t[i].param, t[i].param_bf16, t[i].momentum, t[i].update};
        for (int a = 0; a < 4; ++a) {
            if (!w[a]) continue;
            if (w[a] == t[i].grad) return fail(NOBLE_ERR_INVALID_ARG, "tensor %d: grad is written", i);
            for (int b = 0; b < a; ++b)
                if (w[a] == w[b]) return fail(NOBLE_ERR_INVALID_ARG, "tensor %d: two outputs at one address", i);
            for (int j = 0; j < i; ++j) {
                if (t[j].rows * t[j].cols == 0) continue;
                if (w[a] == t[j].param || w[a] == t[j].param_bf16 || w[a] == t[j].momentum || w[a] == t[j].update ||
                    w[a] == t[j].grad)
                    return fail(NOBLE_ERR_INVALID_ARG, "tensors %d and %d share memory that is written", j, i);
            }
        }
        for (int j = 0; j < i; ++j)
            if (t[j].rows * t[j].cols && (t[i].grad == t[j].param || t[i].grad == t[j].param_bf16 || t[i].grad == t[j].momentum ||
                                          t[i].grad == t[j].update))
                return fail(NOBLE_ERR_INVALID_ARG, "tensors %d and %d share memory that is written", j, i);
    }
    return NOBLE_OK;
}

// Workspace of one launch's matrices: X twice, A and B (each with its low parts if precise),
// partial sums.
struct MuonLayout {
    size_t x[2], a, b, sums, total;
};
int64_t muon_ld(int64_t cols) { return (int64_t)align_up((size_t)cols, 8); }
// Small matrices cost launches, not products, and the error of a small X is not averaged.
bool muon_precise(const noble_muon_tensor &t, uint32_t flags)
{
    return (flags & NOBLE_MUON_PRECISE) != 0 || std::min(t.rows, t.cols) <= 256;
}
MuonLayout muon_layout(const noble_muon_tensor &t, bool precise, size_t at)
{
    MuonLayout w{};
    auto take = [&](size_t bytes) {
        const size_t p = at;
        at = align_up(at + bytes, 256);
        return p;
    };
    const size_t m = (size_t)std::min(t.rows, t.cols), k = (size_t)std::max(t.rows, t.cols), e = precise ? 4 : 2;
    for (size_t &x : w.x) x = take(m * (size_t)muon_ld((int64_t)k) * e);
    w.a = take(m * (size_t)muon_ld((int64_t)m) * e);
    w.b = take(m * (size_t)muon_ld((int64_t)m) * e);
    w.sums = take(muon::kMomentBlocks * sizeof(double));
    w.total = at;
    return w;
}

// The matrices of the next launch: up to kMost that are not empty, from *next on.
int muon_group(const noble_muon_tensor *t, int n, int *next, int (&pick)[muon::kMost])
{
    int got = 0;
    for (; *next < n && got < muon::kMost; ++*next)
        if (t[*next].rows * t[*next].cols > 0) pick[got++] = *next;
    return got;
}

noble_status muon_run(const noble_muon_tensor *t, const int *pick, int n, const noble_muon_hparams *hp, char *ws, cudaStream_t st)
{
    muon::Batch b{};
    b.n = n, b.momentum = hp->momentum, b.eps = hp->eps, b.nesterov = (hp->flags & NOBLE_MUON_NESTEROV) != 0;
    muon::Products pa{}, pb{}, px[2];
    size_t at = 0;
    int tiles = 0, blocks = 0;
    double bytes = 0.0;
    for (int i = 0; i < n; ++i) {
        const noble_muon_tensor &s = t[pick[i]];
        muon::Matrix &M = b.t[i];
        const bool precise = muon_precise(s, hp->flags);
        const MuonLayout w = muon_layout(s, precise, at);
        at = w.total;
        M.param = s.param, M.param_bf16 = static_cast<bf *>(s.param_bf16), M.update = static_cast<bf *>(s.update);
        M.grad = s.grad, M.mom = s.momentum;
        M.n = s.rows * s.cols, M.rows = (int)s.rows, M.cols = (int)s.cols;
        M.tall = s.rows > s.cols;
        M.m = std::min(M.rows, M.cols), M.k = std::max(M.rows, M.cols), M.ld = (int)muon_ld(M.k);
        const float lr = hp->lr * s.lr_mult;
        M.lr = lr * std::sqrt(std::max(1.f, (float)M.rows / (float)M.cols));
        M.decay = s.decay ? lr * hp->weight_decay : 0.f;
        M.sums = reinterpret_cast<double *>(ws + w.sums);
        M.nsums = (int)std::min<int64_t>(muon::kMomentBlocks, ceil_div(M.n, 4096));
        M.tile_begin = tiles, M.tiles_c = (int)ceil_div(M.cols, 64);
        tiles += (int)ceil_div(M.rows, 64) * M.tiles_c;
        blocks = std::max(blocks, M.nsums);
        bytes += (double)M.n * (12 + (s.update ? 2 : 0) + (s.param ? 8 : 0) + (s.param_bf16 ? 2 : 0));

        const int lda = (int)muon_ld(M.m);
        auto half = [&](size_t off) { return reinterpret_cast<__half *>(ws + off); };
        auto low = [&](size_t off, int64_t ld) { return precise ? half(off) + (int64_t)M.m * ld : nullptr; };
        M.x = half(w.x[0]), M.x_lo = low(w.x[0], M.ld);
        M.o = half(w.x[hp->steps % 2]), M.o_lo = low(w.x[hp->steps % 2], M.ld);
        __half *A = half(w.a), *Al = low(w.a, lda), *B = half(w.b), *Bl = low(w.b, lda);
        for (int h = 0; h < 2; ++h) {
            __half *X = half(w.x[h]), *Xl = low(w.x[h], M.ld), *Y = half(w.x[!h]), *Yl = low(w.x[!h], M.ld);
            // X <- B X from this half of the pair into the other
            px[h].p[i] = {B, Bl, X, Xl, nullptr, nullptr, Y, Yl, M.m, M.k, M.m, lda, M.ld, M.ld, 0, 1.f / muon::kScaleB, 0.f, 0.f, 1, 0, 0};
        }
        pa.p[i] = {M.x, M.x_lo, M.x, M.x_lo, nullptr, nullptr, A, Al, M.m, M.m, M.k, M.ld, M.ld, lda, 0,
                   muon::kScaleA / (muon::kScaleX * muon::kScaleX), 0.f, 0.f, 0, 0, 0};
        pb.p[i] = {A, Al, A, Al, A, Al, B, Bl, M.m, M.m, M.m, lda, lda, lda, lda,
                   muon::kC * muon::kScaleB / (muon::kScaleA * muon::kScaleA), muon::kB * muon::kScaleB / muon::kScaleA,
                   muon::kA * muon::kScaleB, 0, 0, 0};
    }
    auto count = [&](muon::Products &g) {
        int total = 0;
        g.n = n;
        for (int i = 0; i < n; ++i) {
            g.p[i].tile_begin = total, g.p[i].tiles_n = (int)ceil_div(g.p[i].n, 64);
            total += (int)ceil_div(g.p[i].m, 64) * g.p[i].tiles_n;
        }
        return total;
    };
    const int ta = count(pa), tb = count(pb), tx = count(px[0]);
    count(px[1]);
    const KernelInfo hbm{"muon_elementwise", kBoundHbm, 0.0, bytes / 3}, mma{"muon_product", kBoundTensor, 0.0, 0.0};
    NOBLE_TRY(run(st, hbm, [&] { muon::momentum_kernel<<<dim3((unsigned)blocks, (unsigned)n), 256, 0, st>>>(b); }));
    NOBLE_TRY(run(st, hbm, [&] { muon::scale_kernel<<<(unsigned)tiles, 256, 0, st>>>(b); }));
    for (int k = 0; k < hp->steps; ++k) {
        const int h = k % 2;
        for (int i = 0; i < n; ++i) {
            pa.p[i].a = pa.p[i].b = px[h].p[i].b;
            pa.p[i].a_lo = pa.p[i].b_lo = px[h].p[i].b_lo;
        }
        NOBLE_TRY(run(st, mma, [&] { muon::product_kernel<<<(unsigned)ta, 256, 0, st>>>(pa); }));
        NOBLE_TRY(run(st, mma, [&] { muon::product_kernel<<<(unsigned)tb, 256, 0, st>>>(pb); }));
        NOBLE_TRY(run(st, mma, [&] { muon::product_kernel<<<(unsigned)tx, 256, 0, st>>>(px[h]); }));
    }
    return run(st, hbm, [&] { muon::apply_kernel<<<(unsigned)tiles, 256, 0, st>>>(b); });
}

}  // namespace
}  // namespace noble

using namespace noble;

extern "C" {

noble_status noble_norm_fwd(const noble_norm_desc *d, const void *x, const void *res, const float *gain, const float *bias,
                            void *sum, void *y, float *stats, noble_stream stream)
{
    g_last_error[0] = 0;
    g_call_kernels = 0;
    NOBLE_TRY(validate(d));
    const bool empty = d->T == 0;
    NOBLE_TRY(check_ptr(x, "x", empty));
    NOBLE_TRY(check_ptr(res, "res", true));
    NOBLE_TRY(check_ptr(gain, "gain", true));
    NOBLE_TRY(check_ptr(bias, "bias", true));
    NOBLE_TRY(check_ptr(sum, "sum", !res));
    NOBLE_TRY(check_ptr(y, "y", empty));
    NOBLE_TRY(check_ptr(stats, "stats", true));
    if (res && sum == y && !empty) return fail(NOBLE_ERR_INVALID_ARG, "sum and y at one address");
    if (empty) return NOBLE_OK;
    NOBLE_TRY(check_device());
    cudaStream_t st = (cudaStream_t)stream;
    return d->dtype == NOBLE_BF16 ? norm_fwd<bf>(d, x, res, gain, bias, sum, y, stats, st)
                                  : norm_fwd<float>(d, x, res, gain, bias, sum, y, stats, st);
}

size_t noble_norm_bwd_workspace_bytes(const noble_norm_desc *d)
{
    if (validate(d) != NOBLE_OK) return 0;
    return std::max<size_t>(256, (size_t)ceil_div(d->T, norm_rows_per_part(d)) * 2 * (size_t)d->d * 4);
}

noble_status noble_norm_bwd(const noble_norm_desc *d, const void *dy, const void *s, const float *stats, const float *gain,
                            const void *dstream, void *dx, float *dgain, float *dbias, void *workspace, size_t workspace_bytes,
                            noble_stream stream)
{
    g_last_error[0] = 0;
    g_call_kernels = 0;
    NOBLE_TRY(validate(d));
    const bool empty = d->T == 0;
    NOBLE_TRY(check_ptr(dy, "dy", empty));
    NOBLE_TRY(check_ptr(s, "s", empty));
    NOBLE_TRY(check_ptr(stats, "stats", empty));
    NOBLE_TRY(check_ptr(gain, "gain", true));
    NOBLE_TRY(check_ptr(dstream, "dstream", true));
    NOBLE_TRY(check_ptr(dx, "dx", empty));
    NOBLE_TRY(check_ptr(dgain, "dgain", true));
    NOBLE_TRY(check_ptr(dbias, "dbias", true));
    if (dgain && dgain == dbias) return fail(NOBLE_ERR_INVALID_ARG, "dgain and dbias at one address");
    NOBLE_TRY(check_workspace(workspace, workspace_bytes, noble_norm_bwd_workspace_bytes(d)));
    NOBLE_TRY(check_device());
    cudaStream_t st = (cudaStream_t)stream;
    if (empty) {
        for (float *p : {dgain, dbias})
            if (p && memset_async(p, 0, (size_t)d->d * 4, st) != cudaSuccess)
                return fail(NOBLE_ERR_CUDA, "memset: %s", cudaGetErrorString(cudaGetLastError()));
        return NOBLE_OK;
    }
    return d->dtype == NOBLE_BF16 ? norm_bwd<bf>(d, dy, s, stats, gain, dstream, dx, dgain, dbias, workspace, st)
                                  : norm_bwd<float>(d, dy, s, stats, gain, dstream, dx, dgain, dbias, workspace, st);
}

noble_status noble_embed_fwd(const noble_embed_desc *d, const int32_t *ids, const void *table, void *y, noble_stream stream)
{
    g_last_error[0] = 0;
    g_call_kernels = 0;
    NOBLE_TRY(validate(d));
    const bool empty = d->T == 0;
    NOBLE_TRY(check_ptr(ids, "ids", empty));
    NOBLE_TRY(check_ptr(table, "table", empty));
    NOBLE_TRY(check_ptr(y, "y", empty));
    if (empty) return NOBLE_OK;
    NOBLE_TRY(check_device());
    cudaStream_t st = (cudaStream_t)stream;
    return d->dtype == NOBLE_BF16 ? embed_fwd<bf>(d, ids, table, y, st) : embed_fwd<float>(d, ids, table, y, st);
}

size_t noble_embed_bwd_workspace_bytes(const noble_embed_desc *d)
{
    return validate(d) == NOBLE_OK ? embed_work(d).total : 0;
}

noble_status noble_embed_bwd(const noble_embed_desc *d, const int32_t *ids, const void *dy, float *dtable, void *workspace,
                             size_t workspace_bytes, noble_stream stream)
{
    g_last_error[0] = 0;
    g_call_kernels = 0;
    NOBLE_TRY(validate(d));
    const bool empty = d->T == 0;
    NOBLE_TRY(check_ptr(ids, "ids", empty));
    NOBLE_TRY(check_ptr(dy, "dy", empty));
    NOBLE_TRY(check_ptr(dtable, "dtable", false));
    NOBLE_TRY(check_workspace(workspace, workspace_bytes, noble_embed_bwd_workspace_bytes(d)));
    NOBLE_TRY(check_device());
    cudaStream_t st = (cudaStream_t)stream;
    if (empty) {
        if (memset_async(dtable, 0, (size_t)d->vocab * (size_t)d->d * 4, st) != cudaSuccess)
            return fail(NOBLE_ERR_CUDA, "memset: %s", cudaGetErrorString(cudaGetLastError()));
        return NOBLE_OK;
    }
    return d->dtype == NOBLE_BF16 ? embed_bwd<bf>(d, ids, dy, dtable, workspace, st)
                                  : embed_bwd<float>(d, ids, dy, dtable, workspace, st);
}

size_t noble_muon_workspace_bytes(const noble_muon_tensor *tensors, int n_tensors, uint32_t flags)
{
    if (validate_muon(tensors, n_tensors, flags) != NOBLE_OK) return 0;
    size_t most = 256;
    int pick[muon::kMost];
    for (int next = 0; next < n_tensors;) {
        size_t at = 0;
        const int n = muon_group(tensors, n_tensors, &next, pick);
        for (int i = 0; i < n; ++i) at = muon_layout(tensors[pick[i]], muon_precise(tensors[pick[i]], flags), at).total;
        most = std::max(most, at);
    }
    return most;
}

noble_status noble_muon_step(const noble_muon_tensor *tensors, int n_tensors, const noble_muon_hparams *hp, void *workspace,
                             size_t workspace_bytes, noble_stream stream)
{
    g_last_error[0] = 0;
    g_call_kernels = 0;
    if (!hp) return fail(NOBLE_ERR_INVALID_ARG, "hparams is NULL");
    NOBLE_TRY(validate_muon(tensors, n_tensors, hp->flags));
    if (!(hp->lr >= 0.f) || !std::isfinite(hp->lr) || !(hp->momentum >= 0.f && hp->momentum < 1.f) ||
        !(hp->weight_decay >= 0.f) || !std::isfinite(hp->weight_decay) || !(hp->eps >= 0.f) || !std::isfinite(hp->eps) ||
        hp->steps < 0 || hp->steps > 16)
        return fail(NOBLE_ERR_INVALID_ARG, "hyperparameters (steps %d)", (int)hp->steps);
    bool work = false;
    for (int i = 0; i < n_tensors; ++i) {
        const noble_muon_tensor &t = tensors[i];
        const bool empty = t.rows * t.cols == 0;
        work |= !empty;
        NOBLE_TRY(check_ptr(t.param, "param", true));
        NOBLE_TRY(check_ptr(t.grad, "grad", empty));
        NOBLE_TRY(check_ptr(t.momentum, "momentum", empty));
        NOBLE_TRY(check_ptr(t.param_bf16, "param_bf16", true));
        NOBLE_TRY(check_ptr(t.update, "update", true));
        if (!empty && !t.param && (t.param_bf16 || !t.update))
            return fail(NOBLE_ERR_INVALID_ARG, t.param_bf16 ? "tensor %d: param_bf16 without param" : "tensor %d: neither param nor update", i);
    }
    NOBLE_TRY(check_apart(tensors, n_tensors));
    if (!work) return NOBLE_OK;
    NOBLE_TRY(check_workspace(workspace, workspace_bytes, noble_muon_workspace_bytes(tensors, n_tensors, hp->flags)));
    NOBLE_TRY(check_device());
    int pick[muon::kMost];
    for (int next = 0; next < n_tensors;) {
        const int n = muon_group(tensors, n_tensors, &next, pick);
        if (n) NOBLE_TRY(muon_run(tensors, pick, n, hp, static_cast<char *>(workspace), (cudaStream_t)stream));
    }
    return NOBLE_OK;
}

}  // extern "C"
