// Optimizer step by orthogonalised momentum, on a group of matrices.
//
//   m <- momentum m + g,   u = g + momentum m (Nesterov) or m
//   X = u / (|u|_F + eps), as its transpose if u has more rows than columns
//   `steps` times:  A = X X^T,  B = a I + b A + c A^2,  X <- B X
//   p <- p - lr decay p - lr sqrt(max(1, rows / columns)) X
//
// The iteration takes every singular value s of X to s (a + b s^2 + c s^4), which brings
// those above about 1 / 500 near 1 within five steps; a, b, c (the quintic of the Muon
// optimizer) are chosen for that and let them end between 0.7 and 1.2.
//
// Matrices of the iteration are held in fp16, scaled by powers of two so that nothing in them
// overflows and small elements keep their 11 bits: |X| <= 1.21 (elements up to 2^15.3 after
// scaling), |A| <= 1.46, |B| <= 3.45.  One rounding to fp16 puts an error of 2^-12 on an
// element; five steps of a matrix with a Gaussian spectrum leave 1e-3 of the norm of
// the result, an eighth of what bf16 would.  "Precise" holds each element as the sum of two
// fp16 numbers (22 bits) and multiplies three products: 1e-6 for 64 x 64, 1e-5 for 8192 x 128 and 4e-5 for
// 2048 x 8192, whose sums in the tensor core are as long.
#pragma once

#include <cuda_fp16.h>

#include "cluster.cuh"

namespace noble {
namespace muon {

constexpr int kMost = 16;  // matrices of a launch
constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
// powers of two that X, A and B are held at
constexpr float kScaleX = 32768.f, kScaleA = 32768.f, kScaleB = 16384.f;

struct Matrix {
    float *param;
    __nv_bfloat16 *param_bf16, *update;
    const float *grad;
    float *mom;
    int64_t n;          // elements
    int rows, cols;
    int m, k, ld, m8;   // of X: rows (the smaller side), columns, elements between rows, rows with padding
    int tall;           // X is the transpose
    float lr, decay;    // lr sqrt(max(1, rows / cols)), lr weight_decay
    __half *x, *x_lo;   // X as the iteration begins; x_lo: low parts (precise)
    __half *x_other, *x_other_lo;  // its other place
    const __half *o, *o_lo;  // ... and ends
    double *sums;       // partial sums of squares of u
    int nsums;
    int tile_begin, tiles_c;  // 64 x 64 tiles of the matrix: first of the launch, tiles of a row
};
struct Batch {
    Matrix t[kMost];
    int n, tiles;       // matrices; 64 x 64 tiles of all
    float momentum, eps;
    int nesterov;
    uint32_t *counts;   // of the products (muon_gemm.cuh), set to zero
    int ncounts;
};

constexpr int kMomentBlocks = 304;  // of a matrix, at most: two per SM

__device__ __forceinline__ float blend(const Batch &b, float g, float m) { return b.nesterov ? fmaf(b.momentum, m, g) : m; }

// New momentum, and partial sums of u^2: fp32 over 16 elements, then fp64.
__global__ void __launch_bounds__(256) momentum_kernel(const __grid_constant__ Batch b)
{
    __shared__ double sm[8];
    ptx::griddep_launch();
    const Matrix &M = b.t[blockIdx.y];
    if ((int)blockIdx.x >= M.nsums) return;
    const int64_t n4 = M.n / 4, stride = (int64_t)M.nsums * 256, first = (int64_t)blockIdx.x * 256 + threadIdx.x;
    double total = 0.0;
    auto one = [&](float g, float &m) {
        m = fmaf(b.momentum, m, g);
        const float u = blend(b, g, m);
        return u * u;
    };
    for (int64_t i = first; i < n4; i += 4 * stride) {
        float4 g[4], m[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int64_t at = i + q * stride;
            g[q] = m[q] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (at < n4) g[q] = reinterpret_cast<const float4 *>(M.grad)[at], m[q] = reinterpret_cast<const float4 *>(M.mom)[at];
        }
        float s = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            s += one(g[q].x, m[q].x);
            s += one(g[q].y, m[q].y);
            s += one(g[q].z, m[q].z);
            s += one(g[q].w, m[q].w);
            if (i + q * stride < n4) reinterpret_cast<float4 *>(M.mom)[i + q * stride] = m[q];
        }
        if (s > 1e-25f && s < 1e37f) {
            total += s;
        } else {  // squares that fp32 does not hold
            auto square = [&](float gi, float mi) {
                const double u = blend(b, gi, mi);
                total += u * u;
            };
#pragma unroll 1
            for (int q = 0; q < 4; ++q) square(g[q].x, m[q].x), square(g[q].y, m[q].y), square(g[q].z, m[q].z), square(g[q].w, m[q].w);
        }
    }
    const int64_t last = 4 * n4 + first;
    if (last < M.n) {
        float m = M.mom[last];
        one(M.grad[last], m);
        const double u = blend(b, M.grad[last], m);
        total += u * u;
        M.mom[last] = m;
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) total += __shfl_xor_sync(0xffffffffu, total, o);
    if (threadIdx.x % 32 == 0) sm[threadIdx.x / 32] = total;
    __syncthreads();
    if (threadIdx.x == 0) {
        total = 0.0;
        for (int w = 0; w < 8; ++w) total += sm[w];
        M.sums[blockIdx.x] = total;
    }
}

// Which matrix a 64 x 64 tile of the launch belongs to.
__device__ __forceinline__ int tile_matrix(const Batch &b, int tile)
{
    int j = 0;
    while (j + 1 < b.n && tile >= b.t[j + 1].tile_begin) ++j;
    return j;
}

// Eight elements of a row, of which the first `n` are there; `wide`: 16-byte accesses are aligned.
__device__ __forceinline__ void load8(const float *p, int n, bool wide, float (&f)[8])
{
    if (wide && n >= 8) {
        const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
        f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = i < n ? p[i] : 0.f;
    }
}
__device__ __forceinline__ void store8(float *p, int n, bool wide, const float (&f)[8])
{
    if (wide && n >= 8) {
        reinterpret_cast<float4 *>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = f[i];
    }
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, int n, bool wide, const float (&f)[8])
{
    if (wide && n >= 8) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(ptx::pack_bf16x2(f[0], f[1]), ptx::pack_bf16x2(f[2], f[3]),
                                                   ptx::pack_bf16x2(f[4], f[5]), ptx::pack_bf16x2(f[6], f[7]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = __float2bfloat16_rn(f[i]);
    }
}
// Rows of X and of the like are padded to whole groups of eight.
__device__ __forceinline__ void store_halves(__half *p, float (&f)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
        const float2 r = __half22float2(h);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
        f[2 * i] -= r.x, f[2 * i + 1] -= r.y;  // what is left
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void add_halves(const __half *p, float (&f)[8])
{
    const uint4 q = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 r = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
        f[2 * i] += r.x, f[2 * i + 1] += r.y;
    }
}

// The 64 x 64 tile at (r0, c0) of a matrix whose rows are not aligned: lanes along a row.
template <class F>
__device__ __forceinline__ void each_element(const Matrix &M, int r0, int c0, F &&f)
{
#pragma unroll 4
    for (int i = threadIdx.x; i < 64 * 64; i += 256) {
        const int r = i / 64, c = i % 64;
        f(r, c, r0 + r < M.rows && c0 + c < M.cols, (int64_t)(r0 + r) * M.cols + c0 + c);
    }
}

// kScaleX / (|u| + eps) as a power of two and the rest: fp32 need not hold it.  NaN where u is not finite,
// an infinite norm among them: times 0 the finite elements would look like a result.
__device__ __forceinline__ float2 inverse_norm(const Matrix &M, float eps)
{
    __shared__ double sm[8];
    __shared__ float2 inv;
    double s = 0.0;
    for (int i = threadIdx.x; i < M.nsums; i += 256) s += M.sums[i];
#pragma unroll
    for (int o = 16; o > 0; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
    __syncthreads();
    if (threadIdx.x % 32 == 0) sm[threadIdx.x / 32] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
        for (int w = 0; w < 8; ++w) s += sm[w];
        const double norm = sqrt(s) + (double)eps;
        const double f = !isfinite(norm) ? (double)NAN : norm > 0.0 ? (double)kScaleX / norm : 0.0;
        const int e = f > 0.0 ? max(-126, min(126, ilogb(f))) : 0;
        inv = make_float2(ldexpf(1.f, e), (float)ldexp(f, -e));
    }
    __syncthreads();
    return inv;
}

// X = u / (|u| + eps) in fp16, in tiles of 64 x 64 elements of u: 512 groups of eight, two per thread.
// Tiles go from the last one to the first; of 2048 x 8192 gradient and momentum are read from DRAM all the same
// (134 MB in 34 us).  Rows that pad X to a
// multiple of eight are zero in both of its places, as the products read them (times zeros).
__global__ void __launch_bounds__(256) scale_kernel(const __grid_constant__ Batch b)
{
    __shared__ float tile[64][65];
    ptx::griddep_launch();
    ptx::griddep_wait();
    for (int i = blockIdx.x * 256 + threadIdx.x; i < b.ncounts; i += gridDim.x * 256) b.counts[i] = 0;
    int last = -1;
    float2 inv = make_float2(0.f, 0.f);
    for (int t = b.tiles - 1 - (int)blockIdx.x; t >= 0; t -= gridDim.x) {
        const int j = tile_matrix(b, t);
        const Matrix &M = b.t[j];
        const int at = t - M.tile_begin, r0 = at / M.tiles_c * 64, c0 = at % M.tiles_c * 64;
        const bool wide = M.cols % 4 == 0;
        float g[2][8], u[2][8];
        if (wide) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int r = r0 + 32 * k + threadIdx.x / 8, c = c0 + threadIdx.x % 8 * 8, n = r < M.rows ? M.cols - c : 0;
                const int64_t e = (int64_t)r * M.cols + c;
                load8(M.mom + e, n, true, u[k]);
                if (b.nesterov) load8(M.grad + e, n, true, g[k]);
            }
        }
        if (at == 0) {
            const int pad = (M.m8 - M.m) * M.ld;
            for (int i = threadIdx.x; i < pad; i += 256) {
                const int64_t e = (int64_t)M.m * M.ld + i;
                M.x[e] = M.x_other[e] = __ushort_as_half(0);
                if (M.x_lo) M.x_lo[e] = M.x_other_lo[e] = __ushort_as_half(0);
            }
        }
        if (j != last) inv = inverse_norm(M, b.eps);
        last = j;
        if (M.tall || !wide) __syncthreads();  // the tile before this one is through
        if (!wide) {
            each_element(M, r0, c0, [&](int r, int c, bool in, int64_t e) {
                tile[r][c] = in ? (b.nesterov ? blend(b, M.grad[e], M.mom[e]) : M.mom[e]) * inv.x * inv.y : 0.f;
            });
        } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int r = 32 * k + threadIdx.x / 8, c = threadIdx.x % 8 * 8;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    u[k][i] = (b.nesterov ? blend(b, g[k][i], u[k][i]) : u[k][i]) * inv.x * inv.y;
                    if (M.tall) tile[r][c + i] = u[k][i];
                }
            }
        }
        if (M.tall || !wide) __syncthreads();
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            // of X: row, column within the tile
            const int r = 32 * k + threadIdx.x / 8, c = threadIdx.x % 8 * 8;
            if (M.tall || !wide)
#pragma unroll
                for (int i = 0; i < 8; ++i) u[k][i] = M.tall ? tile[c + i][r] : tile[r][c + i];
            const int xr = (M.tall ? c0 : r0) + r, xc = (M.tall ? r0 : c0) + c;
            if (xr >= M.m || xc >= M.k) continue;
            const int64_t e = (int64_t)xr * M.ld + xc;
            store_halves(M.x + e, u[k]);
            if (M.x_lo) store_halves(M.x_lo + e, u[k]);
        }
    }
}

// The update, a 64 x 64 tile per block.
__global__ void __launch_bounds__(256) apply_kernel(const __grid_constant__ Batch b)
{
    __shared__ float tile[64][65];
    ptx::griddep_wait();
    const Matrix &M = b.t[tile_matrix(b, blockIdx.x)];
    const int at = blockIdx.x - M.tile_begin, r0 = at / M.tiles_c * 64, c0 = at % M.tiles_c * 64;
    const bool wide = M.cols % 8 == 0;
    float o[2][8], p[2][8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int r = 32 * k + threadIdx.x / 8, c = threadIdx.x % 8 * 8;
        if (M.param && wide) {
            const int n = r0 + r < M.rows ? M.cols - c0 - c : 0;
            load8(M.param + (int64_t)(r0 + r) * M.cols + c0 + c, n, true, p[k]);
        }
        const int xr = (M.tall ? c0 : r0) + r, xc = (M.tall ? r0 : c0) + c;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[k][i] = 0.f;
        if (xr < M.m && xc < M.k) {
            const int64_t e = (int64_t)xr * M.ld + xc;
            add_halves(M.o + e, o[k]);
            if (M.o_lo) add_halves(M.o_lo + e, o[k]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            o[k][i] *= 1.f / kScaleX;
            if (M.tall) tile[c + i][r] = o[k][i];
            else if (!wide) tile[r][c + i] = o[k][i];
        }
    }
    if (M.tall || !wide) __syncthreads();
    if (!wide) {
        each_element(M, r0, c0, [&](int r, int c, bool in, int64_t e) {
            if (!in) return;
            const float x = tile[r][c];
            if (M.update) M.update[e] = __float2bfloat16_rn(x);
            if (!M.param) return;
            float v = M.param[e];
            v = fmaf(-M.lr, x, fmaf(-M.decay, v, v));
            M.param[e] = v;
            if (M.param_bf16) M.param_bf16[e] = __float2bfloat16_rn(v);
        });
        return;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int r = 32 * k + threadIdx.x / 8, c = threadIdx.x % 8 * 8;
        const int n = r0 + r < M.rows ? M.cols - c0 - c : 0;
        if (n <= 0) continue;
        const int64_t e = (int64_t)(r0 + r) * M.cols + c0 + c;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (M.tall) o[k][i] = tile[r][c + i];
        if (M.update) store8(M.update + e, n, true, o[k]);
        if (!M.param) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) p[k][i] = fmaf(-M.lr, o[k][i], fmaf(-M.decay, p[k][i], p[k][i]));
        store8(M.param + e, n, true, p[k]);
        if (M.param_bf16) store8(M.param_bf16 + e, n, true, p[k]);
    }
}

}  // namespace muon
}  // namespace noble
