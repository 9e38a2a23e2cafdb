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
// fp16 numbers (22 bits) and multiplies three products: 1e-6.
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
    int m, k, ld;       // of X: rows (the smaller side), columns, elements between rows
    int tall;           // X is the transpose
    float lr, decay;    // lr sqrt(max(1, rows / cols)), lr weight_decay
    __half *x, *x_lo;   // X as the iteration begins; x_lo: low parts (precise)
    const __half *o, *o_lo;  // ... and ends
    double *sums;       // partial sums of squares of u
    int nsums;
    int tile_begin, tiles_c;  // 64 x 64 tiles of the matrix: first of the launch, tiles of a row
};
struct Batch {
    Matrix t[kMost];
    int n;
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

// X = u / (|u| + eps) in fp16, a 64 x 64 tile of u per block.
__global__ void __launch_bounds__(256) scale_kernel(const __grid_constant__ Batch b)
{
    __shared__ float tile[64][65];
    __shared__ double sm[8];
    __shared__ float inv[2];  // 1 / norm as a power of two and the rest: fp32 need not hold it
    const Matrix &M = b.t[tile_matrix(b, blockIdx.x)];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (int i = blockIdx.x * 256 + threadIdx.x; i < b.ncounts; i += gridDim.x * 256) b.counts[i] = 0;
    // the norm, the same in every block
    double s = 0.0;
    for (int i = threadIdx.x; i < M.nsums; i += 256) s += M.sums[i];
#pragma unroll
    for (int o = 16; o > 0; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) sm[warp] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
        for (int w = 0; w < 8; ++w) s += sm[w];
        const double norm = sqrt(s) + (double)b.eps;
        const double f = norm > 0.0 || norm != norm ? (double)kScaleX / norm : 0.0;
        const int e = f > 0.0 ? max(-126, min(126, ilogb(f))) : 0;
        inv[0] = ldexpf(1.f, e);
        inv[1] = (float)ldexp(f, -e);
    }
    const int at = blockIdx.x - M.tile_begin, r0 = at / M.tiles_c * 64, c0 = at % M.tiles_c * 64;
    for (int i = threadIdx.x; i < 64 * 64; i += 256) {
        const int r = r0 + i / 64, c = c0 + i % 64;
        float u = 0.f;
        if (r < M.rows && c < M.cols) {
            const int64_t e = (int64_t)r * M.cols + c;
            u = blend(b, b.nesterov ? M.grad[e] : 0.f, M.mom[e]);
        }
        tile[i / 64][i % 64] = u;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * 64; i += 256) {
        const int r = i / 64, c = i % 64;  // of X
        const float u = (M.tall ? tile[c][r] : tile[r][c]) * inv[0] * inv[1];
        const int xr = (M.tall ? c0 : r0) + r, xc = (M.tall ? r0 : c0) + c;
        if (xr < M.m && xc < M.k) {
            const __half h = __float2half_rn(u);
            M.x[(int64_t)xr * M.ld + xc] = h;
            if (M.x_lo) M.x_lo[(int64_t)xr * M.ld + xc] = __float2half_rn(u - __half2float(h));
        }
    }
}

// The update, a 64 x 64 tile per block.
__global__ void __launch_bounds__(256) apply_kernel(const __grid_constant__ Batch b)
{
    __shared__ float tile[64][65];
    const Matrix &M = b.t[tile_matrix(b, blockIdx.x)];
    const int at = blockIdx.x - M.tile_begin, r0 = at / M.tiles_c * 64, c0 = at % M.tiles_c * 64;
    for (int i = threadIdx.x; i < 64 * 64; i += 256) {
        const int r = i / 64, c = i % 64;  // of X
        const int xr = (M.tall ? c0 : r0) + r, xc = (M.tall ? r0 : c0) + c;
        float o = 0.f;
        if (xr < M.m && xc < M.k) {
            const int64_t e = (int64_t)xr * M.ld + xc;
            o = __half2float(M.o[e]);
            if (M.o_lo) o += __half2float(M.o_lo[e]);
        }
        if (M.tall) tile[c][r] = o;
        else tile[r][c] = o;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * 64; i += 256) {
        const int r = r0 + i / 64, c = c0 + i % 64;
        if (r >= M.rows || c >= M.cols) continue;
        const int64_t e = (int64_t)r * M.cols + c;
        const float o = tile[i / 64][i % 64] * (1.f / kScaleX);
        if (M.update) M.update[e] = __float2bfloat16_rn(o);
        if (M.param) {
            float p = M.param[e];
            p = fmaf(-M.lr, o, fmaf(-M.decay, p, p));
            M.param[e] = p;
            if (M.param_bf16) M.param_bf16[e] = __float2bfloat16_rn(p);
        }
    }
}

}  // namespace muon
}  // namespace noble
