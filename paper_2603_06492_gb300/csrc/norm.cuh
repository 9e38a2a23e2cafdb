// Layer norm of rows, with the residual stream in front of it, and its gradients.
//
//   s = x + res (rounded to the stream's type), mean and r = 1 / sqrt(var + eps) of s,
//   y = (s - mean) r gain + bias
//   dx = r (w - mean(w) - n mean(w n)) + dstream,   n = (s - mean) r,  w = dy gain
//   dgain = sum over rows of dy n,   dbias = sum over rows of dy
//
// A row stays in the registers of the threads that read it: the variance is the mean square
// of what is left after the mean, and no row is read twice.
#pragma once

#include "cluster.cuh"
#include "common.cuh"

namespace noble {
namespace norm {

// The backward's rows go through a ring in shared memory: a warp of the block keeps it full by bulk
// copies, up to 15 others compute (16 leave 128 registers to each thread).  What bounds the pass is HBM, and rows on their way in
// registers are too few of them beside the sums over rows (50432 x 768 106 us without the ring).
constexpr uint32_t kRingBytes = 200 << 10;  // at most
constexpr int kRingStages = 32;             // at most

// 16 bytes of operands as floats and back
template <typename T> struct Vec;
template <> struct Vec<__nv_bfloat16> {
    static constexpr int n = 8;
    static __device__ __forceinline__ void unpack(const uint4 &q, float (&f)[8])
    {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[2 * i] = __uint_as_float(w[i] << 16), f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8])
    {
        return make_uint4(ptx::pack_bf16x2(f[0], f[1]), ptx::pack_bf16x2(f[2], f[3]), ptx::pack_bf16x2(f[4], f[5]),
                          ptx::pack_bf16x2(f[6], f[7]));
    }
};
template <> struct Vec<float> {
    static constexpr int n = 4;
    static __device__ __forceinline__ void unpack(const uint4 &q, float (&f)[4])
    {
        f[0] = __uint_as_float(q.x), f[1] = __uint_as_float(q.y), f[2] = __uint_as_float(q.z), f[3] = __uint_as_float(q.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[4])
    {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};

template <int N>
__device__ __forceinline__ void load_floats(const float *p, int64_t at, float (&f)[N])
{
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const float4 q = reinterpret_cast<const float4 *>(p + at)[i];
        f[4 * i] = q.x, f[4 * i + 1] = q.y, f[4 * i + 2] = q.z, f[4 * i + 3] = q.w;
    }
}

template <typename T>
struct FwdArgs {
    const T *x, *res;
    const float *gain, *bias;
    T *sum, *y;
    float2 *stats;
    int64_t rows;
    int d, warps, groups;  // warps: of a row; groups: rows of a block at a time
    float eps;
};

// What warps know of their parts of a row: elements, their mean, and the squares off it.
struct Moments {
    float n, mean, squares;
};
__device__ __forceinline__ Moments join(const Moments *p, int warps)
{
    Moments m{0.f, 0.f, 0.f};
    for (int w = 0; w < warps; ++w) m.n += p[w].n, m.mean += p[w].n * p[w].mean;
    m.mean /= m.n;
    for (int w = 0; w < warps; ++w) {
        const float off = p[w].mean - m.mean;
        m.squares += fmaf(p[w].n * off, off, p[w].squares);
    }
    return m;
}

// Blocks of a.groups rows at a time, which take a row after another; the next one's loads are on their
// way while a row is normed.  KEEP: gain and bias stay in registers, or they cost more of L1 than the
// rows (50432 x 768: 33 us).
template <typename T, int NV, bool RES, bool KEEP>
__global__ void __launch_bounds__(512) fwd_kernel(const FwdArgs<T> a)
{
    constexpr int V = Vec<T>::n;
    __shared__ Moments sm[2][16];
    const int step = a.warps * 32, group = threadIdx.x / step, lane = threadIdx.x - group * step, vecs = a.d / V;
    const int64_t stride = (int64_t)gridDim.x * a.groups;
    uint4 q[NV], p[NV];
    auto load = [&](int64_t row) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = i * step + lane;
            q[i] = p[i] = make_uint4(0, 0, 0, 0);
            if (row < a.rows && at < vecs) {
                q[i] = reinterpret_cast<const uint4 *>(a.x + row * a.d)[at];
                if (RES) p[i] = reinterpret_cast<const uint4 *>(a.res + row * a.d)[at];
            }
        }
    };
    auto affine = [&](int i, float (&g)[V], float (&b)[V]) {
#pragma unroll
        for (int j = 0; j < V; ++j) g[j] = 1.f, b[j] = 0.f;
        const int at = i * step + lane;
        if (at < vecs && a.gain) load_floats(a.gain, at * V, g);
        if (at < vecs && a.bias) load_floats(a.bias, at * V, b);
    };
    int64_t row = (int64_t)blockIdx.x * a.groups + group;
    load(row);
    float g[KEEP ? NV : 1][V], b[KEEP ? NV : 1][V];
    if constexpr (KEEP)
#pragma unroll
        for (int i = 0; i < NV; ++i) affine(i, g[i], b[i]);
    int turn = 0;
    // every group of a block goes round as often: there is a barrier among its warps only
    for (int64_t first = (int64_t)blockIdx.x * a.groups; first < a.rows; first += stride, row += stride, turn ^= 1) {
        const bool in = row < a.rows;
        float f[NV][V], sum = 0.f, n = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = i * step + lane;
            Vec<T>::unpack(q[i], f[i]);
            if constexpr (RES) {
                float r[V];
                Vec<T>::unpack(p[i], r);
#pragma unroll
                for (int j = 0; j < V; ++j) f[i][j] += r[j];
                const uint4 s = Vec<T>::pack(f[i]);
                Vec<T>::unpack(s, f[i]);  // the stream as it is stored
                if (in && at < vecs) reinterpret_cast<uint4 *>(a.sum + row * a.d)[at] = s;
            }
            if (at < vecs) n += V;
#pragma unroll
            for (int j = 0; j < V; ++j) sum += f[i][j];
        }
        load(row + stride);
#pragma unroll
        for (int o = 16; o > 0; o /= 2) {
            sum += __shfl_xor_sync(0xffffffffu, sum, o);
            n += __shfl_xor_sync(0xffffffffu, n, o);
        }
        Moments m{n, n > 0.f ? sum / n : 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * step + lane < vecs)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float off = f[i][j] - m.mean;
                    m.squares = fmaf(off, off, m.squares);
                }
#pragma unroll
        for (int o = 16; o > 0; o /= 2) m.squares += __shfl_xor_sync(0xffffffffu, m.squares, o);
        if (a.warps > 1) {
            if (threadIdx.x % 32 == 0) sm[turn][threadIdx.x / 32] = m;
            ptx::named_barrier_sync(1 + group, step);
            m = join(sm[turn] + group * a.warps, a.warps);
        }
        if (!in) continue;
        const float r = 1.f / sqrtf(m.squares / (float)a.d + a.eps);
        if (a.stats && lane == 0) a.stats[row] = make_float2(m.mean, r);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = i * step + lane;
            if (at >= vecs) continue;
            if constexpr (!KEEP) affine(i, g[0], b[0]);
#pragma unroll
            for (int j = 0; j < V; ++j) f[i][j] = fmaf((f[i][j] - m.mean) * r, g[KEEP ? i : 0][j], b[KEEP ? i : 0][j]);
            reinterpret_cast<uint4 *>(a.y + row * a.d)[at] = Vec<T>::pack(f[i]);
        }
    }
}

// A bulk copy of contiguous bytes (a multiple of 16) into shared memory.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes),
                 "r"(bar)
                 : "memory");
}

// The ring's loading thread: rows first .. first + rows of up to three tensors, `groups` of them to a
// stage [tensors][groups][d].
template <typename T, int N>
__device__ __forceinline__ void feed(const T *const (&from)[N], int64_t first, int rows, int groups, int d, int stages, uint32_t base,
                                     uint32_t full0, uint32_t empty0, uint32_t *status)
{
    const uint32_t row_bytes = (uint32_t)d * sizeof(T), tensor_bytes = row_bytes * groups;
    const int steps = (rows + groups - 1) / groups;
    int s = 0, issued = 0;
    uint32_t ph = 0;
    for (; issued < steps; ++issued) {
        if (!ptx::mbar_wait(empty0 + 8 * s, ph ^ 1, status)) break;
        const int64_t row = first + (int64_t)issued * groups;
        const uint32_t n = (uint32_t)min(groups, rows - issued * groups) * row_bytes;
        ptx::mbar_arrive_expect_tx(full0 + 8 * s, n * N);
#pragma unroll
        for (int i = 0; i < N; ++i) bulk_load(base + ((uint32_t)s * N + i) * tensor_bytes, from[i] + row * d, n, full0 + 8 * s);
        if (++s == stages) s = 0, ph ^= 1;
    }
    // no copy may still be landing when the block ends
    for (int k = max(0, issued - stages); k < issued; ++k) ptx::mbar_wait(full0 + 8 * (k % stages), (k / stages) & 1, nullptr);
}

// Rows that a group of the backward has in hand, by the columns of a thread.
__host__ __device__ constexpr int rows_side_by_side(int columns) { return columns <= 8 ? 2 : 1; }

template <typename T>
struct BwdArgs {
    const T *dy, *s, *dstream;
    const float2 *stats;
    const float *gain;
    T *dx;
    float *part;  // [parts][2][d], or NULL: no gradients of gain and bias
    uint32_t *status;
    int64_t rows;
    int d, warps, groups, rows_per_part;  // warps: of a row; groups: rows at a time
    int stages;
    float inv_d;
};

// Block p takes the rows of part p, R groups' of them at a time.  A thread has the same columns of
// every row, whose sums for dgain and dbias it keeps in registers and the block then adds up in
// order of the groups.  R: rows of a group side by side, for narrow rows, whose chain of loads, sums
// over the row and stores is longer than their work.  WARPS: 15 or, where a row takes more, 16, which leave 96
// registers to a thread: wide rows spill, most of them beyond 8192 columns (4096 rows of bf16: 7680 columns 59 us, 8192
// 64, 8200 166; 2048 of 16384 132).
template <typename T, int NV, bool STREAM, int WARPS>
__global__ void __launch_bounds__(32 * (WARPS + 1), 1) bwd_kernel(const BwdArgs<T> a)
{
    constexpr int V = Vec<T>::n, kTensors = STREAM ? 3 : 2, R = rows_side_by_side(NV * V);
    extern __shared__ __align__(128) uint8_t ring[];  // [stages][tensors][R groups][d], then the sums over rows
    __shared__ float2 sm[2][R][WARPS];
    __shared__ __align__(8) uint64_t bars[2 * kRingStages];
    ptx::griddep_launch();
    const int warp = threadIdx.x / 32, work_warps = a.warps * a.groups, batch = R * a.groups;
    const int64_t first = (int64_t)blockIdx.x * a.rows_per_part;
    const int rows = (int)min((int64_t)a.rows_per_part, a.rows - first), steps = (rows + batch - 1) / batch;
    const uint32_t row_bytes = (uint32_t)a.d * sizeof(T), tensor_bytes = row_bytes * batch;
    const uint32_t full0 = ptx::smem_u32(bars), empty0 = full0 + 8 * kRingStages;
    if (threadIdx.x == 0) {
        for (int i = 0; i < a.stages; ++i) {
            ptx::mbar_init(full0 + 8 * i, 1);
            ptx::mbar_init(empty0 + 8 * i, work_warps);
        }
        ptx::fence_barrier_init();
    }
    __syncthreads();
    const int vecs = a.d / V, per_row = a.warps * 32, tid = threadIdx.x;
    const int group = tid / per_row, lane = tid - group * per_row;
    float dg[NV][V], db[NV][V];
    if (warp == work_warps) {
        if (tid % 32 == 0) {
            if constexpr (STREAM) {
                const T *const from[3] = {a.dy, a.s, a.dstream};
                feed(from, first, rows, batch, a.d, a.stages, ptx::smem_u32(ring), full0, empty0, a.status);
            } else {
                const T *const from[2] = {a.dy, a.s};
                feed(from, first, rows, batch, a.d, a.stages, ptx::smem_u32(ring), full0, empty0, a.status);
            }
        }
    } else if (warp < work_warps) {
        float g[NV][V];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < V; ++j) dg[i][j] = db[i][j] = 0.f, g[i][j] = 1.f;
            if (a.gain && i * per_row + lane < vecs) load_floats(a.gain, (i * per_row + lane) * V, g[i]);
        }
        int s = 0;
        uint32_t ph = 0;
        bool ok = true;
        auto stats = [&](int k, int h) {  // of row h of this group in step k
            const int row = k * batch + h * a.groups + group;
            return row < rows ? a.stats[first + row] : make_float2(0.f, 0.f);
        };
        float2 st[R];
#pragma unroll
        for (int h = 0; h < R; ++h) st[h] = stats(0, h);
        for (int k = 0; k < steps; ++k) {
            float2 next[R];  // the next rows' statistics, a step ahead
#pragma unroll
            for (int h = 0; h < R; ++h) next[h] = stats(k + 1, h);
            // a wait that gave up is reported; the barriers below still need every warp
            if (ok) ok = ptx::mbar_wait(full0 + 8 * s, ph, a.status);
            const uint8_t *at = ring + (size_t)s * kTensors * tensor_bytes + group * row_bytes;
            uint4 qy[R][NV], qs[R][NV];
            float2 t[R];
#pragma unroll
            for (int h = 0; h < R; ++h) {
                t[h] = make_float2(0.f, 0.f);
                const bool in = k * batch + h * a.groups + group < rows;
                const uint8_t *row = at + h * a.groups * row_bytes;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = i * per_row + lane;
                    if (!in || c >= vecs) continue;
                    qy[h][i] = reinterpret_cast<const uint4 *>(row)[c];
                    qs[h][i] = reinterpret_cast<const uint4 *>(row + tensor_bytes)[c];
                    float y[V], n[V];
                    Vec<T>::unpack(qy[h][i], y);
                    Vec<T>::unpack(qs[h][i], n);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        n[j] = (n[j] - st[h].x) * st[h].y;
                        dg[i][j] = fmaf(y[j], n[j], dg[i][j]);
                        db[i][j] += y[j];
                        const float w = y[j] * g[i][j];
                        t[h].x += w;
                        t[h].y = fmaf(w, n[j], t[h].y);
                    }
                }
            }
#pragma unroll
            for (int o = 16; o > 0; o /= 2)
#pragma unroll
                for (int h = 0; h < R; ++h) {
                    t[h].x += __shfl_xor_sync(0xffffffffu, t[h].x, o);
                    t[h].y += __shfl_xor_sync(0xffffffffu, t[h].y, o);
                }
            if (a.warps > 1) {
#pragma unroll
                for (int h = 0; h < R; ++h)
                    if (tid % 32 == 0) sm[k & 1][h][warp] = t[h];
                ptx::named_barrier_sync(1 + group, per_row);
#pragma unroll
                for (int h = 0; h < R; ++h) {
                    t[h] = make_float2(0.f, 0.f);
                    for (int w = 0; w < a.warps; ++w) {
                        const float2 p = sm[k & 1][h][group * a.warps + w];
                        t[h].x += p.x, t[h].y += p.y;
                    }
                }
            }
#pragma unroll
            for (int h = 0; h < R; ++h) {
                const int r = k * batch + h * a.groups + group;
                const float mw = t[h].x * a.inv_d, mwn = t[h].y * a.inv_d;
                T *dx = a.dx + (first + r) * a.d;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = i * per_row + lane;
                    if (r >= rows || c >= vecs) continue;
                    float y[V], n[V];
                    Vec<T>::unpack(qy[h][i], y);
                    Vec<T>::unpack(qs[h][i], n);
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        y[j] = st[h].y * (fmaf(y[j], g[i][j], -mw) - (n[j] - st[h].x) * st[h].y * mwn);
                    if (STREAM) {
                        float e[V];
                        Vec<T>::unpack(reinterpret_cast<const uint4 *>(at + h * a.groups * row_bytes + 2 * tensor_bytes)[c], e);
#pragma unroll
                        for (int j = 0; j < V; ++j) y[j] += e[j];
                    }
                    reinterpret_cast<uint4 *>(dx)[c] = Vec<T>::pack(y);
                }
                st[h] = next[h];
            }
            __syncwarp();
            if (tid % 32 == 0) ptx::mbar_arrive(empty0 + 8 * s);
            if (++s == a.stages) s = 0, ph ^= 1;
        }
    }
    if (!a.part) return;
    float *out = a.part + (int64_t)blockIdx.x * 2 * a.d;
    if (a.groups == 1) {
        if (warp < work_warps)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i * per_row + lane < vecs)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        out[(i * per_row + lane) * V + j] = dg[i][j];
                        out[a.d + (i * per_row + lane) * V + j] = db[i][j];
                    }
        return;
    }
    __syncthreads();  // the ring is through
    float *cols = reinterpret_cast<float *>(ring);  // [groups][2][d]
    if (warp < work_warps)
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * per_row + lane < vecs)
#pragma unroll
                for (int j = 0; j < V; j += 4) {
                    float *to = cols + group * 2 * a.d + (i * per_row + lane) * V + j;
                    *reinterpret_cast<float4 *>(to) = make_float4(dg[i][j], dg[i][j + 1], dg[i][j + 2], dg[i][j + 3]);
                    *reinterpret_cast<float4 *>(to + a.d) = make_float4(db[i][j], db[i][j + 1], db[i][j + 2], db[i][j + 3]);
                }
    __syncthreads();
    for (int c = tid; c < 2 * a.d; c += blockDim.x) {
        float v = 0.f;
        for (int k = 0; k < a.groups; ++k) v += cols[k * 2 * a.d + c];
        out[c] = v;
    }
}

// dgain and dbias from the parts: 32 columns to a block, a range of the parts to each warp, in order;
// then the ranges in order.  Columns 0 to d are dgain's, the others dbias's; either may be NULL.
__global__ void __launch_bounds__(1024) join_kernel(const float *part, int parts, int d, float *dgain, float *dbias)
{
    __shared__ float sm[32][33];
    ptx::griddep_wait();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, col = blockIdx.x * 32 + lane, per = (parts + 31) / 32;
    float v = 0.f;
    if (col < 2 * d) {
        const int end = min(parts, (warp + 1) * per);
#pragma unroll 8
        for (int p = warp * per; p < end; ++p) v += part[(int64_t)p * 2 * d + col];
    }
    sm[warp][lane] = v;
    __syncthreads();
    if (warp != 0 || col >= 2 * d) return;
    v = 0.f;
#pragma unroll
    for (int w = 0; w < 32; ++w) v += sm[w][lane];
    float *out = col < d ? dgain : dbias;
    if (out) out[col < d ? col : col - d] = v;
}

}  // namespace norm
}  // namespace noble
