// What comes before the products of the orthogonalisation: momentum, the Frobenius norm, and X = U / (||U||_F + eps) as high
// and low halves, short side first.
#pragma once

#include "coded.cuh"
#include "gemm.cuh"

namespace rtopk {
namespace mat {

constexpr int kNormBlocks = 256;   // at most this many partial sums of squares per matrix

struct Source {
  const void* src;       // U, or g of the update
  int bf16;
  int64_t ld, stride;
  float* v;              // update: momentum, replaced by mu v + g; null: U is src
  int64_t v_ld, v_stride;
  float mu;
  int nesterov;
  int m, n;
  float eps;
  double* part;          // [batch][kNormBlocks]
  int parts;
};

__device__ __forceinline__ float source_at(const Source& s, int64_t i) {
  return s.bf16 ? __bfloat162float(((const __nv_bfloat16*)s.src)[i]) : ((const float*)s.src)[i];
}
// u from the momentum after its update
__device__ __forceinline__ float update_of(const Source& s, float g, float v) { return s.nesterov ? fmaf(s.mu, v, g) : v; }

// Sums of squares, in binary64 so that neither large nor small gradients leave the range; one partial sum per block, added
// up in a fixed order by the readers.
__global__ void __launch_bounds__(256) k_norm(const __grid_constant__ Source s) {
  __shared__ double part[8];
  const int z = blockIdx.y;
  launch_next();
  double sum = 0.0;
  const int64_t count = (int64_t)s.m * s.n, step = (int64_t)gridDim.x * 256;
  for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < count; k += step) {
    const int64_t r = k / s.n, c = k - r * s.n;
    float u = source_at(s, z * s.stride + r * s.ld + c);
    if (s.v) {
      float* v = s.v + z * s.v_stride + r * s.v_ld + c;
      const float nv = (float)((double)s.mu * (double)*v + (double)u);
      *v = nv;
      u = update_of(s, u, nv);
    }
    sum += (double)u * (double)u;
  }
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0;
    for (int i = 0; i < 8; ++i) sum += part[i];
    s.part[z * kNormBlocks + blockIdx.x] = sum;
  }
}

// One element of X as its halves; the warp's 32 neighbours of a row give one partial sum of squares.
__device__ __forceinline__ void split_store(float u, bool in, __half* hi, __half* lo, float* sum) {
  if (in) {
    const __half h = to_half(u);
    *hi = h;
    *lo = to_half((u - __half2float(h)) * kLoScale);
  }
  u *= u;
#pragma unroll
  for (int o = 16; o; o >>= 1) u += __shfl_xor_sync(0xFFFFFFFFu, u, o);
  if ((threadIdx.x & 31) == 0) *sum = u;
}

// X, 64 x 64 elements of U per block, transposed when U is tall.
__global__ void __launch_bounds__(256)
k_split(const __grid_constant__ Source s, __half* hi, __half* lo, int64_t ld, int64_t stride, float* row_sums, int slots, int64_t d_stride, int transpose) {
  __shared__ float tile[64][65];
  __shared__ float inv_s;
  const int z = blockIdx.z, c0 = blockIdx.x * 64, r0 = blockIdx.y * 64;
  launch_wait();
  launch_next();
  if (threadIdx.x < 32) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < s.parts; i += 32) sum += s.part[z * kNormBlocks + i];
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (threadIdx.x == 0) inv_s = sum == 0.0 ? 0.f : (float)((double)kXScale / (sqrt(sum) + (double)s.eps));
  }
  __syncthreads();
  const float inv = inv_s;
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
  hi += z * stride, lo += z * stride, row_sums += (int64_t)z * slots * d_stride;
  for (int r = y; r < 64; r += 4) {
    const int row = r0 + r, col = c0 + x;
    float u = 0.f;
    if (row < s.m && col < s.n) {
      u = source_at(s, z * s.stride + row * s.ld + col);
      if (s.v) u = update_of(s, u, s.v[z * s.v_stride + row * s.v_ld + col]);
      u *= inv;
    }
    if (transpose) tile[x][r] = u;
    else if (row < s.m && (col & ~31) < s.n) split_store(u, col < s.n, hi + row * ld + col, lo + row * ld + col, row_sums + (col / 32) * d_stride + row);
  }
  if (!transpose) return;
  __syncthreads();
  for (int c = y; c < 64; c += 4) {
    const int row = c0 + c, col = r0 + x;      // of X
    if (row < s.n && (col & ~31) < s.m) split_store(tile[c][x], col < s.m, hi + row * ld + col, lo + row * ld + col, row_sums + (col / 32) * d_stride + row);
  }
}

// Small matrices (the shorter side at most kSmall): the whole operator in one block per matrix, everything in shared memory
// and binary32.  A chain of launches would spend its time starting them: at 64 x 64 a step's three products are
// 1.6 million operations.  X is held transposed, [long][64], so that all products read rows of 64.
constexpr int kSmall = 64;

struct SmallOut {
  float* w;                // update: the weights; null: out
  void* out;
  int bf16;
  int64_t ld, stride;
  float keep, rate;
  float coef[3 * 64];
  int steps;
};

// acc[i][j] += sum_k p[k][i0 + i] q[k][j0 + j], rows of kSmall floats
__device__ __forceinline__ void small_product(const float* p, const float* q, int depth, int i0, int j0, float (&acc)[4][4]) {
#pragma unroll 4
  for (int k = 0; k < depth; ++k) {
    const float4 a = *(const float4*)(p + k * kSmall + i0), b = *(const float4*)(q + k * kSmall + j0);
    const float av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(av[i], bv[j], acc[i][j]);
  }
}

__global__ void __launch_bounds__(256) k_orth_small(const __grid_constant__ Source s, const __grid_constant__ SmallOut to, int transpose) {
  extern __shared__ float small_smem[];
  __shared__ double part[8];
  const int z = blockIdx.x, t = threadIdx.x;
  const int ns = transpose ? s.n : s.m, nl = transpose ? s.m : s.n;
  const int rows = (nl + 7) & ~7;             // both halves of a warp have rows to work on, or neither
  float* x = small_smem;                          // [rows][64]
  float* g = x + rows * kSmall;                   // [64][64]
  float* b = g + kSmall * kSmall;
  for (int i = t; i < rows * kSmall; i += 256) x[i] = 0.f;
  __syncthreads();
  double sum = 0.0;
  for (int k = t; k < s.m * s.n; k += 256) {
    const int r = k / s.n, c = k - r * s.n;
    float u = source_at(s, z * s.stride + r * s.ld + c);
    if (s.v) {
      float* v = s.v + z * s.v_stride + r * s.v_ld + c;
      const float nv = (float)((double)s.mu * (double)*v + (double)u);
      *v = nv;
      u = update_of(s, u, nv);
    }
    sum += (double)u * (double)u;
    x[transpose ? r * kSmall + c : c * kSmall + r] = u;
  }
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if ((t & 31) == 0) part[t >> 5] = sum;
  __syncthreads();
  sum = 0.0;
  for (int i = 0; i < 8; ++i) sum += part[i];
  const float inv = sum == 0.0 ? 0.f : (float)(1.0 / (sqrt(sum) + (double)s.eps));
  for (int i = t; i < rows * kSmall; i += 256) x[i] *= inv;
  __syncthreads();
  const int i0 = (t & 15) * 4, j0 = (t >> 4) * 4;
  for (int step = 0; step < to.steps; ++step) {
    const float ca = to.coef[3 * step], cb = to.coef[3 * step + 1], cc = to.coef[3 * step + 2];
    {
      float acc[4][4] = {};
      small_product(x, x, nl, i0, j0, acc);
#pragma unroll
      for (int j = 0; j < 4; ++j) *(float4*)(g + (j0 + j) * kSmall + i0) = make_float4(acc[0][j], acc[1][j], acc[2][j], acc[3][j]);
    }
    __syncthreads();
    {
      float acc[4][4] = {};
      small_product(g, g, ns, i0, j0, acc);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float4 a = *(const float4*)(g + (j0 + j) * kSmall + i0);
        const float av[4] = {a.x, a.y, a.z, a.w};
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = cc * acc[i][j] + cb * av[i] + (i0 + i == j0 + j ? ca : 0.f);
        *(float4*)(b + (j0 + j) * kSmall + i0) = make_float4(v[0], v[1], v[2], v[3]);
      }
    }
    __syncthreads();
    // a thread's four rows of X are read by its whole group of 16 before they are written: the rows of one group belong to
    // one half of a warp
    for (int r0 = (t >> 4) * 4; r0 < rows; r0 += 64) {
      float acc[4][4] = {};
      for (int k = 0; k < ns; k += 4) {
        float4 xr[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) xr[j] = *(const float4*)(x + (r0 + j) * kSmall + k);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          const float4 p = *(const float4*)(b + (k + kk) * kSmall + i0);
          const float pv[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float xv = kk == 0 ? xr[j].x : kk == 1 ? xr[j].y : kk == 2 ? xr[j].z : xr[j].w;
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i][j] = fmaf(pv[i], xv, acc[i][j]);
          }
        }
      }
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 4; ++j) *(float4*)(x + (r0 + j) * kSmall + i0) = make_float4(acc[0][j], acc[1][j], acc[2][j], acc[3][j]);
      __syncwarp();
    }
    __syncthreads();
  }
  for (int k = t; k < s.m * s.n; k += 256) {
    const int r = k / s.n, c = k - r * s.n;
    const float v = x[transpose ? r * kSmall + c : c * kSmall + r];
    const int64_t at = z * to.stride + r * to.ld + c;
    if (to.w) to.w[at] = to.keep * to.w[at] - to.rate * v;
    else if (to.bf16) ((__nv_bfloat16*)to.out)[at] = __float2bfloat16_rn(v);
    else ((float*)to.out)[at] = v;
  }
}

}  // namespace mat
}  // namespace rtopk
