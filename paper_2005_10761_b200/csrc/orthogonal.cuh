// What comes before the products of the orthogonalisation: momentum, the Frobenius norm, and X = U / (||U||_F + eps) in
// 32 and in 16 bits, short side first.
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
  int vec, v_vec;        // rows allow loads of four
  float eps;
  double* part;          // [batch][kNormBlocks]
  int parts;
};

__device__ __forceinline__ float source_at(const Source& s, int64_t i) {
  return s.bf16 ? __bfloat162float(((const __nv_bfloat16*)s.src)[i]) : ((const float*)s.src)[i];
}
// u from the momentum after its update
__device__ __forceinline__ float update_of(const Source& s, float g, float v) { return s.nesterov ? fmaf(s.mu, v, g) : v; }

// Four neighbours of a row, those past its end zero.
__device__ __forceinline__ float4 load4(const float* p, int left, bool vec) {
  if (vec && left >= 4) return *(const float4*)p;
  return make_float4(left > 0 ? p[0] : 0.f, left > 1 ? p[1] : 0.f, left > 2 ? p[2] : 0.f, left > 3 ? p[3] : 0.f);
}
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p, int left, bool vec) {
  if (vec && left >= 4) {
    const uint2 a = *(const uint2*)p;
    return make_float4(__uint_as_float(a.x << 16), __uint_as_float(a.x & 0xFFFF0000u), __uint_as_float(a.y << 16), __uint_as_float(a.y & 0xFFFF0000u));
  }
  return make_float4(left > 0 ? widen(p[0]) : 0.f, left > 1 ? widen(p[1]) : 0.f, left > 2 ? widen(p[2]) : 0.f, left > 3 ? widen(p[3]) : 0.f);
}
__device__ __forceinline__ float4 source4(const Source& s, int64_t i, int left) {
  return s.bf16 ? load4((const __nv_bfloat16*)s.src + i, left, s.vec) : load4((const float*)s.src + i, left, s.vec);
}

// Sums of squares, in binary64 so that neither large nor small gradients leave the range; one partial sum per block, added
// up in a fixed order by the readers.  A warp takes 1024 neighbours of a row at a time.
constexpr int kNormSpan = 1024;
__global__ void __launch_bounds__(256) k_norm(const __grid_constant__ Source s) {
  __shared__ double part[8];
  const int z = blockIdx.y, lane = threadIdx.x & 31;
  launch_wait();
  launch_next();
  const int pieces = (s.n + kNormSpan - 1) / kNormSpan;
  const int64_t units = (int64_t)s.m * pieces;
  double sum = 0.0;
  for (int64_t k = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); k < units; k += (int64_t)gridDim.x * 8) {
    const int64_t r = k / pieces;
    const int c0 = (int)(k - r * pieces) * kNormSpan + lane * 4;
    const int64_t at = z * s.stride + r * s.ld, at_v = z * s.v_stride + r * s.v_ld;
    float4 u[8], v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = c0 + i * 128;
      u[i] = c < s.n ? source4(s, at + c, s.n - c) : make_float4(0.f, 0.f, 0.f, 0.f);
      if (s.v) v[i] = c < s.n ? load4(s.v + at_v + c, s.n - c, s.v_vec) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = c0 + i * 128, left = s.n - c;
      if (left <= 0) break;
      if (s.v) {
        const float4 g = u[i];
        const float4 nv = make_float4(fmaf(s.mu, v[i].x, g.x), fmaf(s.mu, v[i].y, g.y), fmaf(s.mu, v[i].z, g.z), fmaf(s.mu, v[i].w, g.w));
        float* p = s.v + at_v + c;
        if (s.v_vec && left >= 4) {
          *(float4*)p = nv;
        } else {
          p[0] = nv.x;
          if (left > 1) p[1] = nv.y;
          if (left > 2) p[2] = nv.z;
          if (left > 3) p[3] = nv.w;
        }
        u[i] = make_float4(update_of(s, g.x, nv.x), update_of(s, g.y, nv.y), update_of(s, g.z, nv.z), update_of(s, g.w, nv.w));
      }
      sum += (double)u[i].x * (double)u[i].x;
      sum += (double)u[i].y * (double)u[i].y;
      sum += (double)u[i].z * (double)u[i].z;
      sum += (double)u[i].w * (double)u[i].w;
    }
  }
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if (lane == 0) part[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0;
    for (int i = 0; i < 8; ++i) sum += part[i];
    s.part[z * kNormBlocks + blockIdx.x] = sum;
  }
}

// X, 64 x 64 elements of U per block, transposed when U is tall.  A thread writes eight neighbours of a row of X; four threads together give one partial sum of squares.
__global__ void __launch_bounds__(256)
k_split(const __grid_constant__ Source s, float* x, __half* h, int64_t ld, int64_t stride, float* row_sums, int slots, int64_t d_stride, int transpose) {
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
  {
    const int c = (threadIdx.x & 15) * 4, left = s.n - c0 - c;
    float4 u[4], v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = r0 + (threadIdx.x >> 4) + 16 * i;
      const bool in = r < s.m && left > 0;
      u[i] = in ? source4(s, z * s.stride + r * s.ld + c0 + c, left) : make_float4(0.f, 0.f, 0.f, 0.f);
      if (s.v) v[i] = in ? load4(s.v + z * s.v_stride + r * s.v_ld + c0 + c, left, s.v_vec) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (s.v) u[i] = make_float4(update_of(s, u[i].x, v[i].x), update_of(s, u[i].y, v[i].y), update_of(s, u[i].z, v[i].z), update_of(s, u[i].w, v[i].w));
      float* t = tile[(threadIdx.x >> 4) + 16 * i] + c;
      t[0] = u[i].x, t[1] = u[i].y, t[2] = u[i].z, t[3] = u[i].w;
    }
  }
  __syncthreads();
  const float inv = inv_s;
  x += z * stride, h += z * stride, row_sums += (int64_t)z * slots * d_stride;
  const int ns = transpose ? s.n : s.m, nl = transpose ? s.m : s.n;
  const int a0 = transpose ? c0 : r0, b0 = transpose ? r0 : c0;      // of X: rows and columns
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int a = (threadIdx.x >> 3) + 32 * i, b = (threadIdx.x & 7) * 8;
    float u[8], sum = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      u[j] = (transpose ? tile[b + j][a] : tile[a][b + j]) * inv;
      sum = fmaf(u[j], u[j], sum);
    }
    sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1);
    sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 2);
    if (a0 + a >= ns || b0 + (b & ~31) >= nl) continue;
    if ((b & 31) == 0) row_sums[(int64_t)((b0 + b) / 32) * d_stride + a0 + a] = sum;
    if (b0 + b < nl) {      // the rows' padding takes whole vectors
      const int64_t at = (a0 + a) * ld + b0 + b;
      *(float4*)(x + at) = make_float4(u[0], u[1], u[2], u[3]);
      *(float4*)(x + at + 4) = make_float4(u[4], u[5], u[6], u[7]);
      store_half8(h + at, u);
    }
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
  launch_wait();
  launch_next();
  __syncthreads();
  double sum = 0.0;
  for (int k = t; k < s.m * s.n; k += 256) {
    const int r = k / s.n, c = k - r * s.n;
    float u = source_at(s, z * s.stride + r * s.ld + c);
    if (s.v) {
      float* v = s.v + z * s.v_stride + r * s.v_ld + c;
      const float nv = fmaf(s.mu, *v, u);
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
