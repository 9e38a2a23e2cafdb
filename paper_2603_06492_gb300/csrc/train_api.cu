// C-ABI entry points around the projections of a training step (declared in
// include/noble.h): layer norm, embedding, optimizer step by orthogonalised momentum.
//
// Host side only: argument checks, workspaces and kernel dispatch.
#include <algorithm>
#include <cmath>

#include "host.cuh"
#include "embed.cuh"
#include "muon_small.cuh"
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

// Dynamic shared memory beyond 48 KB has to be allowed for each kernel, in each context; a kernel is
// allowed the same number of bytes every time.
template <class Kern>
noble_status allow_shared(Kern kern, size_t bytes)
{
    struct Done {
        const void *kern;
        CUcontext ctx;
    };
    static std::mutex mu;
    static Done done[64];  // kernels of one signature
    static int n = 0;
    const CUcontext ctx = current_context();
    std::lock_guard<std::mutex> g(mu);
    for (int i = 0; ctx && i < n; ++i)
        if (done[i].kern == (const void *)kern && done[i].ctx == ctx) return NOBLE_OK;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess)
        return fail(NOBLE_ERR_CUDA, "shared memory: %s", cudaGetErrorString(cudaGetLastError()));
    if (n < 64) done[n++] = {(const void *)kern, current_context()};
    return NOBLE_OK;
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

template <typename T>
noble_status norm_fwd(const noble_norm_desc *d, const void *x, const void *res, const float *gain, const float *bias,
                      void *sum, void *y, float *stats, cudaStream_t st)
{
    norm::FwdArgs<T> a{};
    a.x = static_cast<const T *>(x), a.res = static_cast<const T *>(res), a.gain = gain, a.bias = bias;
    a.sum = static_cast<T *>(sum), a.y = static_cast<T *>(y), a.stats = reinterpret_cast<float2 *>(stats);
    a.rows = d->T, a.d = (int)d->d;
    // eps 0: a row of equal elements gives 0 times a finite factor
    a.eps = std::max(d->eps, 1e-37f);
    const KernelInfo ki{"norm_fwd", kBoundHbm, 0.0, (double)sizeof(T) * d->T * d->d * (res ? 4 : 2)};
    const int vecs = (int)(d->d / norm::Vec<T>::n);
    constexpr int kMost = 32 / norm::Vec<T>::n;  // vectors of a thread
    // a warp per row as far as 32 elements a lane go; where there are few rows, eight warps a row
    const int least = (int)ceil_div(vecs, 32 * kMost);
    a.warps = d->T < 4 * kSms ? std::max(least, std::min(8, (int)ceil_div(vecs, 32))) : least;
    a.groups = std::max(1, 8 / a.warps);
    const int nv = (int)ceil_div(vecs, 32 * a.warps);
    auto with = [&](auto n) {
        constexpr bool kKeep = n.value * norm::Vec<T>::n <= 24;
        // as many blocks as an SM's registers hold
        constexpr int kBlocks = n.value * norm::Vec<T>::n >= 16 ? 2 : 4;
        const dim3 grid((unsigned)std::min<int64_t>(ceil_div(d->T, a.groups), kBlocks * kSms)), block(32 * a.warps * a.groups);
        return run(st, ki, [&] {
            if (res) norm::fwd_kernel<T, n.value, true, kKeep><<<grid, block, 0, st>>>(a);
            else norm::fwd_kernel<T, n.value, false, kKeep><<<grid, block, 0, st>>>(a);
        });
    };
    constexpr int kStep = kMost / 4;
    switch (ceil_div(nv, kStep)) {
    case 1: return with(std::integral_constant<int, kStep>{});
    case 2: return with(std::integral_constant<int, 2 * kStep>{});
    case 3: return with(std::integral_constant<int, 3 * kStep>{});
    default: return with(std::integral_constant<int, 4 * kStep>{});
    }
}

// Rows of a part of the sums for dgain and dbias: a block per SM, and at most 512, so that sums of
// like rows stay short.  Beyond 77824 rows the blocks are more than the SMs, and whole parts in a last round that they do
// not fill cost as much as a full one (rows of 768: 77824, and one more, in 68 us, 5.3 TB/s; 98304 in 122, 131072 in 123,
// 160000 in 176).
int norm_rows_per_part(const noble_norm_desc *d)
{
    return (int)std::max<int64_t>(1, std::min<int64_t>(512, ceil_div(d->T, kSms)));
}

template <typename T>
noble_status norm_bwd(const noble_norm_desc *d, const void *dy, const void *s, const float *stats, const float *gain,
                      const void *dstream, void *dx, float *dgain, float *dbias, void *workspace, cudaStream_t st)
{
    norm::BwdArgs<T> a{};
    a.dy = static_cast<const T *>(dy), a.s = static_cast<const T *>(s), a.dstream = static_cast<const T *>(dstream);
    a.stats = reinterpret_cast<const float2 *>(stats), a.gain = gain, a.dx = static_cast<T *>(dx);
    a.part = dgain || dbias ? static_cast<float *>(workspace) : nullptr;
    NOBLE_TRY(get_status(&a.status));
    a.rows = d->T, a.d = (int)d->d, a.rows_per_part = norm_rows_per_part(d), a.inv_d = 1.f / (float)d->d;
    const int64_t parts = ceil_div(d->T, a.rows_per_part);
    const KernelInfo ki{"norm_bwd", kBoundHbm, 0.0, (double)sizeof(T) * d->T * d->d * (dstream ? 4 : 3)};
    // columns of a thread: 16, or 8 where fewer lanes then stay idle; of bf16 24 where a warp then has a
    // row to itself (50432 x 768: 46 us, with 8 columns 59); 32 where 16 warps reach no further
    const int vecs = a.d / norm::Vec<T>::n;
    constexpr int kOne = 16 / norm::Vec<T>::n, kWide = 3 * kOne / 2;
    const int warps1 = (int)ceil_div(vecs, 32 * kOne / 2), warps2 = (int)ceil_div(vecs, 32 * kOne);
    const int per = warps2 > 16                                            ? 2 * kOne
                    : sizeof(T) == 2 && warps2 == 2 && vecs <= 32 * kWide ? kWide
                    : warps1 <= 15 && warps1 < 2 * warps2                 ? kOne / 2
                                                                          : kOne;
    a.warps = (int)ceil_div(vecs, 32 * per);
    const int side = norm::rows_side_by_side(per * norm::Vec<T>::n);
    a.groups = std::max(1, std::min<int>(15 / a.warps, (int)ceil_div(a.rows_per_part, side)));
    const uint32_t stage = (uint32_t)(side * a.groups) * (uint32_t)a.d * (uint32_t)sizeof(T) * (dstream ? 3 : 2);
    a.stages = (int)std::max<uint32_t>(1, std::min<uint32_t>({norm::kRingBytes / stage, (uint32_t)norm::kRingStages,
                                                              (uint32_t)ceil_div(a.rows_per_part, side * a.groups)}));
    const size_t smem = std::max<size_t>((size_t)a.stages * stage, a.groups > 1 ? (size_t)a.groups * 2 * a.d * 4 : 0);
    auto launch = [&](auto kern) -> noble_status {
        NOBLE_TRY(allow_shared(kern, norm::kRingBytes));
        return run(st, ki, [&] { kern<<<(unsigned)parts, 32 * (a.warps * a.groups + 1), smem, st>>>(a); });
    };
    auto with = [&](auto nv, auto warps) {
        return dstream ? launch(norm::bwd_kernel<T, nv.value, true, warps.value>) : launch(norm::bwd_kernel<T, nv.value, false, warps.value>);
    };
    const std::integral_constant<int, 15> most{};
    const std::integral_constant<int, 16> more{};
    if (per == kOne / 2) NOBLE_TRY(with(std::integral_constant<int, kOne / 2>{}, most));
    else if (per == kWide) NOBLE_TRY(with(std::integral_constant<int, sizeof(T) == 2 ? kWide : kOne>{}, most));
    else if (per == 2 * kOne) NOBLE_TRY(with(std::integral_constant<int, 2 * kOne>{}, more));
    else if (a.warps == 16) NOBLE_TRY(with(std::integral_constant<int, kOne>{}, more));
    else NOBLE_TRY(with(std::integral_constant<int, kOne>{}, most));
    if (!a.part) return NOBLE_OK;
    const bool pdl = pdl_ok();
    return run(st, {"norm_join", kBoundHbm, 0.0, 8.0 * parts * d->d}, [&] {
        launch_maybe_pdl(norm::join_kernel, dim3((unsigned)ceil_div(2 * d->d, 32)), dim3(1024), 0, st, pdl, (const float *)a.part, (int)parts,
                         a.d, dgain, dbias);
    });
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
    size_t count, head, begin, rank, list, long_row, piece, piece_part, joined, part, total;
};
// One launch for few tokens that do not share rows too much: its blocks look for their rows among all
// of them (512 tokens of text, 5000 x 256: 10 us, by lists 20; 100 x 256: 29 and 20).
bool embed_few(const noble_embed_desc *d) { return d->T <= 64 || (d->T <= embed::kFewTokens && 2 * d->T <= d->vocab); }
EmbedWork embed_work(const noble_embed_desc *d)
{
    EmbedWork w{};
    if (embed_few(d)) {
        w.total = 256;
        return w;
    }
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t p = at;
        at = align_up(at + bytes, 256);
        return p;
    };
    // a long list has more than kShort tokens, and no more pieces than a (kShort + 1)th of them; one of
    // several pieces has more than kPiece tokens, and fewer pieces than a 32nd of them
    const size_t T = (size_t)d->T, V = (size_t)d->vocab, lists = T / (embed::kShort + 1) + 1, parts = T / (embed::kPiece / 2) + 1;
    w.head = take(32);
    w.count = take(4 * V);
    w.begin = take(4 * V);
    w.rank = take(4 * T);
    w.list = take(4 * T);
    w.long_row = take(4 * lists);
    w.piece = take(8 * lists);
    w.piece_part = take(4 * lists);
    w.joined = take(8 * (T / embed::kPiece + 1));
    w.part = take(4 * parts * (size_t)d->d);
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
    a.wide = reinterpret_cast<uintptr_t>(dtable) % 32 == 0;
    NOBLE_TRY(get_status(&a.status));
    const int vecs = (int)(d->d / norm::Vec<T>::n);
    const unsigned slices = (unsigned)ceil_div(vecs, 32);
    const double out = 4.0 * d->vocab * d->d, in = (double)sizeof(T) * d->T * d->d;
    if (embed_few(d))
        return run(st, {"embed_few", kBoundHbm, 0.0, in + out}, [&] {
            embed::few_kernel<T><<<dim3((unsigned)ceil_div(d->vocab, embed::kFewRows), slices), 256, 0, st>>>(a);
        });
    const EmbedWork w = embed_work(d);
    char *ws = static_cast<char *>(workspace);
    auto at = [&](size_t off) { return reinterpret_cast<uint32_t *>(ws + off); };
    a.head = at(w.head), a.count = at(w.count), a.begin = at(w.begin), a.rank = at(w.rank), a.list = at(w.list);
    a.long_row = at(w.long_row), a.piece_part = at(w.piece_part), a.joined = reinterpret_cast<uint2 *>(ws + w.joined);
    a.piece = reinterpret_cast<uint2 *>(ws + w.piece), a.part = reinterpret_cast<float *>(ws + w.part);
    a.part_wide = reinterpret_cast<uintptr_t>(a.part) % 32 == 0;
    const KernelInfo index{"embed_index", kBoundHbm, 0.0, 0.0}, sum{"embed_sum", kBoundHbm, 0.0, in + out};
    const auto launch = [&](const KernelInfo &ki, auto kern, dim3 grid, size_t smem, unsigned threads = 256) {
        const bool pdl = pdl_ok();
        return run(st, ki, [&] { launch_maybe_pdl(kern, grid, dim3(threads), smem, st, pdl, a); });
    };
    const unsigned lists = (unsigned)(d->T / (embed::kShort + 1));
    const size_t bits = (size_t)std::min<int64_t>(embed::kWindow, (int64_t)align_up((size_t)d->T, 32)) / 8;
    if (d->T <= embed::kIndexTokens && d->vocab <= embed::kIndexRows) {
        NOBLE_TRY(launch(index, embed::index_kernel<T>, dim3(embed::kIndexBlocks), 0, embed::kIndexThreads));
    } else {
        if (memset_async(ws, 0, w.count + 4 * (size_t)d->vocab, st) != cudaSuccess)
            return fail(NOBLE_ERR_CUDA, "memset: %s", cudaGetErrorString(cudaGetLastError()));
        const unsigned per_token = (unsigned)ceil_div(d->T, 256);
        NOBLE_TRY(launch(index, embed::count_kernel<T>, dim3(per_token), 0));
        NOBLE_TRY(launch(index, embed::lists_kernel<T>, dim3((unsigned)ceil_div(d->vocab, 8 * 256)), 0));
        NOBLE_TRY(launch(index, embed::place_kernel<T>, dim3(per_token), 0));
    }
    NOBLE_TRY(launch(index, embed::order_kernel<T>, dim3(std::min(lists, 4u * kSms)), bits));
    // rows of a warp: two, where there are that many for 16 warps per SM (8192 tokens, 50257 x 1024, and 65536,
    // 131072 x 2048: one 80 and 509 us, two 67 and 302, four 68 and 309); pieces of long lists come first
    a.rows_per_warp = (int)std::max<int64_t>(1, std::min<int64_t>(2, d->vocab / (16 * kSms)));
    a.piece_blocks = (int)std::min<int64_t>(ceil_div((int64_t)lists * slices, 8), 4 * kSms);
    const int64_t blocks = a.piece_blocks + ceil_div(d->vocab, 8 * a.rows_per_warp);
    // columns in parts where rows alone are too few warps
    const unsigned parts = a.rows_per_warp > 1 ? 1 : std::min(slices, 64u);
    NOBLE_TRY(launch(sum, embed::sum_kernel<T>, dim3((unsigned)blocks, parts), 0));
    return launch(sum, embed::join_kernel<T>, dim3((unsigned)std::min<int64_t>(ceil_div(d->T, embed::kPiece), kSms), (unsigned)std::min<int64_t>(ceil_div(d->d, 128), 64)), 0);
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

// Small matrices cost launches, not products, and the error of a small X is not averaged: pairs without being
// asked.  That costs nothing up to 128 rows and 2048 columns, which iterate in one launch (128 x 2048 78 us, without
// pairs by launches 129), and most from there on: 129 x 2048 182 us (without 136), 256 x 1024 183 (129); 300 x 1024,
// not in pairs, takes 130.
bool muon_precise(const noble_muon_tensor &t, uint32_t flags)
{
    return (flags & NOBLE_MUON_PRECISE) != 0 || std::min(t.rows, t.cols) <= 256;
}
// Elements between rows of X, A and B; X also has whole groups of eight rows (make_half_map4).
int64_t muon_ld(int64_t cols) { return (int64_t)align_up((size_t)cols, 64); }

// The three products of a step, in this order: A = X X^T, B = a I + b A + c A A, X <- B X.
enum { kGram, kPoly, kNext, kPhases };

// A group of up to kMost matrices: their places in the workspace, and how each product is cut
// into units.  The shapes decide, so that results are the same on every device.
struct MuonPlan {
    int n;
    int pick[muon::kMost];
    struct {
        size_t x[2], a, b, sums;
    } at[muon::kMost];
    size_t counts, part, total;
    int ncounts;
    int small;  // blocks of a matrix if all iterate in one launch, else 0
    muon::mma::Problem p[kPhases][muon::kMost];  // sizes only
    int order[kPhases][muon::kMost];             // place in the launch -> matrix
    int units[kPhases];
};

// Tiles of a problem with tiles of bn columns.
int muon_tiles(const muon::mma::Problem &p, int bn)
{
    const int tm = (int)ceil_div(p.m, muon::mma::kRows), tn = (int)ceil_div(p.n, bn);
    return p.sym ? muon::mma::sym_tiles_before(tm, tn, muon::mma::kRows / bn) : tm * tn;
}
// Times of a unit in k-blocks of a tile of 256 columns, 0.29 us, of its main loop and of its epilogue, which
// runs beside the next unit's main loop.  That is the tensor pipe's rate; one k-block of 128 columns takes 0.27 us
// all the same, for three quarters of the operands.  Parts of a split K are stored, fenced and joined, which takes longer than most main loops:
// splits pay only while all units run at once (X X^T of 1024 x 4096, 76 pairs: 20 tiles of 128 columns whole, in 3
// and in 4 parts 6, 0 and 5 us above the best; 2048 x 8192: 36 tiles of 256 columns whole and in 2 parts 7 and 0;
// B X of 2048 x 8192, 256 tiles, whole and in 2 parts 0 and 70).
double muon_main(int kb, int bn) { return kb * (bn == 256 ? 1.0 : 0.92) + 2; }
double muon_epilogue(int bn, int nsplit)
{
    if (nsplit == 1) return bn == 256 ? 12 : 6;
    return (bn == 256 ? 2 : 1) * (20 + 1.1 * nsplit);
}

// Columns of tiles and splits of K for the problems of a launch, by the time of the busiest pair: the
// problem with the most work in 1, 2, ... parts while they all run at once, the others in parts as long
// as its, or twice or four times that.
void muon_cut(muon::mma::Problem *p, int *order, int n, int *units)
{
    using namespace muon::mma;
    int main = 0;
    auto work = [&](int i) { return (int64_t)muon_tiles(p[i], 256) * p[i].kb * p[i].segs; };
    for (int i = 1; i < n; ++i)
        if (work(i) > work(main)) main = i;
    const int main_kb = p[main].kb * p[main].segs;
    double best = 1e300;
    Problem kept[muon::kMost];
    int kept_order[muon::kMost], kept_units = 0;
    auto attempt = [&](int bn, int splits, int longer) {
        const int most = (int)ceil_div(main_kb, splits);  // k-blocks of a unit
        for (int i = 0; i < n; ++i) {
            Problem &q = p[i];
            const int kb = q.kb * q.segs;
            q.bn = q.n <= 128 ? 128 : bn;
            q.tiles_m = (int)ceil_div(q.m, kRows), q.tiles_n = (int)ceil_div(q.n, q.bn);
            q.kb_per_split = (int)ceil_div(kb, std::min<int64_t>(kMostSplits, ceil_div(kb, i == main ? most : longer * most)));
            q.nsplit = (int)ceil_div(kb, q.kb_per_split);
            order[i] = i;
        }
        std::sort(order, order + n, [&](int a, int b) {
            const double x = muon_main(p[a].kb_per_split, p[a].bn), y = muon_main(p[b].kb_per_split, p[b].bn);
            return x != y ? x > y : a < b;
        });
        double load[kPairs] = {}, longest = 0.0;
        int total = 0;
        for (int k = 0; k < n; ++k) {
            Problem &q = p[order[k]];
            q.unit_begin = total;
            const int count = muon_tiles(q, q.bn) * q.nsplit;
            const double loop = muon_main(q.kb_per_split, q.bn), end = muon_epilogue(q.bn, q.nsplit);
            auto add = [&](int pair, int units) {
                load[pair] += std::max(loop, end) * units;
                longest = std::max(longest, load[pair] + std::min(loop, end));
            };
            // whole rounds of all pairs, then the units that are left in their places
            const int rounds = count / kPairs;
            for (int c = 0; rounds && c < kPairs; ++c) add(c, rounds);
            for (int c = rounds * kPairs; c < count; ++c) add(pair_of(total + c, kPairs), 1);
            total += count;
        }
        if (longest < best) {
            best = longest;
            std::copy(p, p + n, kept), std::copy(order, order + n, kept_order);
            kept_units = total;
        }
    };
    for (int bn : {256, 128})
        for (int splits = 1; splits <= kMostSplits; ++splits) {
            if (splits > 1 && (splits > main_kb || muon_tiles(p[main], bn) * splits > kPairs)) break;
            for (int longer : {1, 2, 4}) {
                if (longer > 1 && n == 1) break;
                attempt(bn, splits, longer);
            }
        }
    std::copy(kept, kept + n, p), std::copy(kept_order, kept_order + n, order);
    *units = kept_units;
    // pieces of the accumulation of pairs: the columns of TMEM that a unit has, all 512 where no pair takes a
    // second one
    for (int i = 0; i < n; ++i) {
        const int pieces = p[i].segs > 1 ? (kept_units <= kPairs ? 512 : 256) / p[i].bn : 1;
        p[i].piece_kb = (int)align_up((size_t)ceil_div(p[i].kb_per_split, pieces), 2);
    }
}

// Blocks per matrix of a group whose matrices all iterate in one launch (muon_small.cuh), or 0.  Eight, or
// four where they hold few columns each: 128 x 1024 62 us a call in a graph with eight and 72 with four, 128 x 512
// 58 and 60, 64 x 64 35 and 33.  A GB300 does not hold more than some 14 clusters of eight at once: 16 of 64 x 1024
// take 54 us with four blocks each, 73 with eight; 8 of them 52 and 43.
int muon_small(const noble_muon_tensor *t, const int *pick, int n)
{
    int64_t most = 0;
    for (int i = 0; i < n; ++i) {
        if (std::min(t[pick[i]].rows, t[pick[i]].cols) > muon::small::kRows) return 0;
        most = std::max({most, t[pick[i]].rows, t[pick[i]].cols});
    }
    if (most > muon::small::kBlocks * muon::small::kCols) return 0;
    if (n == 0) return 0;
    return most <= 512 || (n > 8 && most <= 1024) ? muon::small::kFewBlocks : muon::small::kBlocks;
}

// Takes the next matrices that are not empty, from *next on.
MuonPlan muon_plan(const noble_muon_tensor *t, int n, int *next, uint32_t flags)
{
    MuonPlan w{};
    for (; *next < n && w.n < muon::kMost; ++*next)
        if (t[*next].rows * t[*next].cols > 0) w.pick[w.n++] = *next;
    auto take = [&](size_t bytes) {
        const size_t p = w.total;
        w.total = align_up(w.total + bytes, 256);
        return p;
    };
    w.small = muon_small(t, w.pick, w.n);
    for (int i = 0; i < w.n; ++i) {
        const noble_muon_tensor &s = t[w.pick[i]];
        const bool precise = muon_precise(s, flags);
        const int m = (int)std::min(s.rows, s.cols), k = (int)std::max(s.rows, s.cols);
        const size_t e = precise ? 4 : 2;
        for (size_t &x : w.at[i].x) x = take(align_up((size_t)m, 8) * (size_t)muon_ld(k) * e);
        if (!w.small) {
            w.at[i].a = take((size_t)m * (size_t)muon_ld(m) * e);
            w.at[i].b = take((size_t)m * (size_t)muon_ld(m) * e);
        }
        w.at[i].sums = take(muon::kMomentBlocks * sizeof(double));
        for (int j = 0; j < kPhases; ++j) {
            muon::mma::Problem &p = w.p[j][i];
            p.m = m, p.n = j == kNext ? k : m;
            p.kb = (int)ceil_div(j == kGram ? k : m, muon::mma::kBK);
            p.segs = precise ? 3 : 1, p.pairs = precise;
            p.sym = j != kNext, p.b_mn = j == kNext;
        }
    }
    if (w.small) return w;
    size_t part = 0;
    for (int j = 0; j < kPhases; ++j) {
        muon_cut(w.p[j], w.order[j], w.n, &w.units[j]);
        size_t bytes = 0;
        int counts = 0;
        for (int i = 0; i < w.n; ++i) {
            muon::mma::Problem &p = w.p[j][i];
            if (p.nsplit == 1) continue;
            const size_t tiles = (size_t)muon_tiles(p, p.bn);
            bytes += tiles * p.nsplit * muon::mma::kRows * p.bn * 4;
            counts += (int)tiles * 64;
        }
        part = std::max(part, bytes), w.ncounts = std::max(w.ncounts, counts);
    }
    w.counts = take((size_t)w.ncounts * 4);
    w.part = take(part);
    return w;
}

// TMA map of an fp16 matrix: boxes of 64 or 32 columns, with the swizzle of that width.
noble_status make_half_map(CUtensorMap *m, const __half *p, int rows, int cols, int64_t ld, uint32_t box_rows, uint32_t box_cols = 64)
{
    EncodeTiledFn enc = encode_fn();
    if (!enc) return fail(NOBLE_ERR_CUDA, "cuTensorMapEncodeTiled is unavailable");
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
    cuuint32_t box[2] = {box_cols, box_rows};
    cuuint32_t estr[2] = {1, 1};
    const CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<__half *>(p), dims, strides, box, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS)
        return fail(NOBLE_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d): rows=%d cols=%d ld=%lld", (int)r, rows, cols, (long long)ld);
    return NOBLE_OK;
}

// The 4-D map of X as the operand that is not along K (make_map_mn4 of noble_api.cu has the
// layout): whole groups of eight rows, the last filled up with zeros, and of 64 columns.  A 2-D map of
// boxes of 64 rows makes the products 1.4 times slower (0.37 us a k-block of 256 x 256, not 0.26).
noble_status make_half_map4(CUtensorMap *m, const __half *p, int rows, int64_t ld, uint32_t chunks)
{
    EncodeTiledFn enc = encode_fn();
    if (!enc) return fail(NOBLE_ERR_CUDA, "cuTensorMapEncodeTiled is unavailable");
    const cuuint64_t pitch = (cuuint64_t)ld * 2;
    cuuint64_t dims[4] = {64, 8, (cuuint64_t)ld / 64, (cuuint64_t)ceil_div(rows, 8)};
    cuuint64_t strides[3] = {pitch, 128, 8 * pitch};
    cuuint32_t box[4] = {64, 8, chunks, 8};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    const CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<__half *>(p), dims, strides, box, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(NOBLE_ERR_CUDA, "cuTensorMapEncodeTiled (4-D) failed (%d): rows=%d ld=%lld", (int)r, rows, (long long)ld);
    return NOBLE_OK;
}

// A matrix of the iteration: its high parts, and low parts behind them or NULL.
struct HalfMatrix {
    __half *hi, *lo;
    int rows, cols;
    int64_t ld;
    noble_status maps4(CUtensorMap *m, uint32_t chunks) const
    {
        NOBLE_TRY(make_half_map4(m, hi, rows, ld, chunks));
        return lo ? make_half_map4(m + 1, lo, rows, ld, chunks) : NOBLE_OK;
    }
    noble_status store_maps(CUtensorMap *m) const
    {
        NOBLE_TRY(make_half_map(m, hi, rows, cols, ld, 32, 32));
        return lo ? make_half_map(m + 1, lo, rows, cols, ld, 32, 32) : NOBLE_OK;
    }
    noble_status maps(CUtensorMap *m, uint32_t box_rows) const
    {
        NOBLE_TRY(make_half_map(m, hi, rows, cols, ld, box_rows));
        return lo ? make_half_map(m + 1, lo, rows, cols, ld, box_rows) : NOBLE_OK;
    }
};

template <int N, bool WIDE>
noble_status muon_product(const muon::mma::Args<N> &g, const KernelInfo &ki, cudaStream_t st)
{
    constexpr size_t smem = muon::mma::Smem<WIDE>::kDynamic;
    NOBLE_TRY(allow_shared(muon::mma::product_pairs<N, WIDE>, smem));
    // each pair takes units of its own: no pair waits for another, so that they need not all be resident
    const int pairs = std::min(g.units, muon::mma::kPairs);
    const bool pdl = pdl_ok();
    return run(st, ki, [&] {
        launch_maybe_pdl(muon::mma::product_pairs<N, WIDE>, dim3(2 * (unsigned)pairs), dim3(tc::pair::kPairThreads), smem, st, pdl, g);
    });
}

noble_status muon_iterate(const muon::Batch &b, const MuonPlan &w, int steps, cudaStream_t st)
{
    using namespace muon::small;
    Args g{};
    g.b = b, g.steps = steps;
    NOBLE_TRY(get_status(&g.status));
    double flops = 0.0;
    for (int i = 0; i < b.n; ++i) {
        g.cols[i] = (int)align_up((size_t)ceil_div(b.t[i].k, w.small), 64);
        flops += steps * (double)b.t[i].m * b.t[i].m * (3.0 * b.t[i].k + b.t[i].m);
    }
    NOBLE_TRY(allow_shared(iterate_kernel, kDynamic));
    const bool pdl = pdl_ok();
    return run(st, {"muon_iterate", kBoundTensor, flops, 0.0}, [&] {
        launch_cluster(iterate_kernel, dim3((unsigned)(b.n * w.small)), w.small, dim3(kThreads), kDynamic, st, pdl, g);
    });
}

template <int N>
noble_status muon_run(const noble_muon_tensor *t, const MuonPlan &w, const noble_muon_hparams *hp, char *ws, cudaStream_t st)
{
    using Args = muon::mma::Args<N>;
    bool wide[kPhases] = {};
    muon::Batch b{};
    b.n = w.n, b.momentum = hp->momentum, b.eps = hp->eps, b.nesterov = (hp->flags & NOBLE_MUON_NESTEROV) != 0;
    b.counts = reinterpret_cast<uint32_t *>(ws + w.counts), b.ncounts = w.ncounts;
    HalfMatrix X[2][muon::kMost], A[muon::kMost], B[muon::kMost];
    int tiles = 0, blocks = 0;
    double bytes = 0.0;
    for (int i = 0; i < w.n; ++i) {
        const noble_muon_tensor &s = t[w.pick[i]];
        muon::Matrix &M = b.t[i];
        const bool precise = w.p[kGram][i].pairs != 0;
        M.param = s.param, M.param_bf16 = static_cast<bf *>(s.param_bf16), M.update = static_cast<bf *>(s.update);
        M.grad = s.grad, M.mom = s.momentum;
        M.n = s.rows * s.cols, M.rows = (int)s.rows, M.cols = (int)s.cols;
        M.tall = s.rows > s.cols;
        M.m = std::min(M.rows, M.cols), M.k = std::max(M.rows, M.cols), M.ld = (int)muon_ld(M.k);
        M.m8 = (int)align_up((size_t)M.m, 8);
        const float lr = hp->lr * s.lr_mult;
        M.lr = lr * std::sqrt(std::max(1.f, (float)M.rows / (float)M.cols));
        M.decay = s.decay ? lr * hp->weight_decay : 0.f;
        M.sums = reinterpret_cast<double *>(ws + w.at[i].sums);
        M.nsums = (int)std::min<int64_t>(muon::kMomentBlocks, ceil_div(M.n, 4096));
        M.tile_begin = tiles, M.tiles_c = (int)ceil_div(M.cols, 64);
        tiles += (int)ceil_div(M.rows, 64) * M.tiles_c;
        blocks = std::max(blocks, M.nsums);
        bytes += (double)M.n * (12 + (s.update ? 2 : 0) + (s.param ? 8 : 0) + (s.param_bf16 ? 2 : 0));
        auto matrix = [&](size_t off, int rows, int cols) {
            const int64_t ld = muon_ld(cols);
            __half *p = reinterpret_cast<__half *>(ws + off);
            return HalfMatrix{p, precise ? p + rows * ld : nullptr, M.m, cols, ld};
        };
        for (int h = 0; h < 2; ++h) X[h][i] = matrix(w.at[i].x[h], M.m8, M.k);
        A[i] = matrix(w.at[i].a, M.m, M.m), B[i] = matrix(w.at[i].b, M.m, M.m);
        M.x = X[0][i].hi, M.x_lo = X[0][i].lo, M.x_other = X[1][i].hi, M.x_other_lo = X[1][i].lo;
        M.o = X[hp->steps % 2][i].hi, M.o_lo = X[hp->steps % 2][i].lo;
    }
    b.tiles = tiles;
    // a product's arguments: what it multiplies, what it writes
    double flops[kPhases] = {};
    auto arguments = [&](Args &g, int phase, int half) -> noble_status {
        g.n = w.n, g.units = w.units[phase];
        NOBLE_TRY(get_status(&g.status));
        size_t part = w.part;
        uint32_t *count = b.counts;
        flops[phase] = 0.0;
        for (int k = 0; k < w.n; ++k) {
            const int i = w.order[phase][k];
            muon::mma::Problem &p = g.p[k];
            CUtensorMap *m = g.map[k];
            p = w.p[phase][i];
            const uint32_t rows = (uint32_t)p.bn / 2;
            wide[phase] |= p.bn == 256;
            if (phase == kGram) {
                NOBLE_TRY(X[half][i].maps(m, 128));
                NOBLE_TRY(X[half][i].maps(m + 2, rows));
                NOBLE_TRY(A[i].store_maps(m + 4));
                p.alpha = muon::kScaleA / (muon::kScaleX * muon::kScaleX);
            } else if (phase == kPoly) {
                NOBLE_TRY(A[i].maps(m, 128));
                NOBLE_TRY(A[i].maps(m + 2, rows));
                NOBLE_TRY(B[i].store_maps(m + 4));
                p.alpha = muon::kC * muon::kScaleB / (muon::kScaleA * muon::kScaleA);
                p.beta = muon::kB * muon::kScaleB / muon::kScaleA, p.diag = muon::kA * muon::kScaleB;
                p.d = A[i].hi, p.d_lo = A[i].lo, p.ldd = (int)A[i].ld;
            } else {
                NOBLE_TRY(B[i].maps(m, 128));
                NOBLE_TRY(X[half][i].maps4(m + 2, rows / 64));
                NOBLE_TRY(X[!half][i].store_maps(m + 4));
                p.alpha = 1.f / muon::kScaleB;
            }
            flops[phase] += 2.0 * p.m * p.n * (phase == kGram ? b.t[i].k : p.m) * (p.sym ? 0.5 : 1.0);
            if (p.nsplit > 1) {
                const int n = muon_tiles(p, p.bn);
                p.part = reinterpret_cast<float *>(ws + part), p.count = count;
                part += (size_t)n * p.nsplit * muon::mma::kRows * p.bn * 4;
                count += n * 64;
            }
        }
        return NOBLE_OK;
    };
    const KernelInfo hbm{"muon_elementwise", kBoundHbm, 0.0, bytes / 3};
    NOBLE_TRY(run(st, hbm, [&] { muon::momentum_kernel<<<dim3((unsigned)blocks, (unsigned)w.n), 256, 0, st>>>(b); }));
    const auto dependent = [&](auto kern, int grid) {
        const bool pdl = pdl_ok();
        return run(st, hbm, [&] { launch_maybe_pdl(kern, dim3((unsigned)grid), dim3(256), 0, st, pdl, b); });
    };
    NOBLE_TRY(dependent(muon::scale_kernel, std::min(tiles, 4 * kSms)));
    if (w.small) {
        if (hp->steps > 0) NOBLE_TRY(muon_iterate(b, w, hp->steps, st));
        return dependent(muon::apply_kernel, tiles);
    }
    Args gram[2] = {}, poly = {}, next[2] = {};
    auto product = [&](const Args &g, int phase) {
        static const char *const names[kPhases] = {"muon_gram", "muon_poly", "muon_next"};
        const KernelInfo ki{names[phase], kBoundTensor, flops[phase], 0.0};
        return wide[phase] ? muon_product<N, true>(g, ki, st) : muon_product<N, false>(g, ki, st);
    };
    for (int k = 0; k < hp->steps; ++k) {
        const int h = k % 2;
        if (k < 2) NOBLE_TRY(arguments(gram[h], kGram, h));
        NOBLE_TRY(product(gram[h], kGram));
        if (k == 0) NOBLE_TRY(arguments(poly, kPoly, 0));
        NOBLE_TRY(product(poly, kPoly));
        if (k < 2) NOBLE_TRY(arguments(next[h], kNext, h));
        NOBLE_TRY(product(next[h], kNext));
    }
    return dependent(muon::apply_kernel, tiles);
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
    for (int next = 0; next < n_tensors;) most = std::max(most, muon_plan(tensors, n_tensors, &next, flags).total);
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
    // all groups' plans fit before anything is enqueued; a single group's is kept
    MuonPlan plan{};
    int next = 0;
    size_t need = 256;
    while (next < n_tensors) {
        plan = muon_plan(tensors, n_tensors, &next, hp->flags);
        need = std::max(need, plan.total);
    }
    NOBLE_TRY(check_workspace(workspace, workspace_bytes, need));
    NOBLE_TRY(check_device());
    auto go = [&](const MuonPlan &w) {
        char *ws = static_cast<char *>(workspace);
        return w.n <= 4 ? muon_run<4>(tensors, w, hp, ws, (cudaStream_t)stream) : muon_run<muon::kMost>(tensors, w, hp, ws, (cudaStream_t)stream);
    };
    if (n_tensors <= muon::kMost) return go(plan);
    for (next = 0; next < n_tensors;) {
        const MuonPlan w = muon_plan(tensors, n_tensors, &next, hp->flags);
        if (w.n) NOBLE_TRY(go(w));
    }
    return NOBLE_OK;
}

}  // extern "C"
