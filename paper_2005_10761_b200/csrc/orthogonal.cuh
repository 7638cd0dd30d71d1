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

// Small matrices (the shorter side at most 64, the longer at most 256): the whole operator in one block per matrix, everything in
// shared memory.  A chain of launches would spend its time starting them: at 64 x 64 a step's three products are 1.6 million
// operations.  What bounds this kernel is the chain of dependent products inside one SM, so they are mma.sync products of the
// block's sixteen warps, 16 x 16 entries each, with no trip through tensor memory between them.  Every factor is the sum of two
// 16-bit numbers, high and low, and three of the four partial products are formed: 2^-21 of the result is lost, so
// that a matrix too small for errors to average out is as exact as a large one.
constexpr int kSmall = 64, kSmallLong = 256, kSmallThreads = 512;
constexpr int kSmallKeep = kSmall * kSmallLong / kSmallThreads;      // elements of U in a thread's registers
constexpr int kSmallLd = kSmall + 8;
constexpr float kSmallScale = 32.f;                                  // of X, its Gram matrix and the polynomial

struct SmallOut {
  float* w;                // update: the weights; null: out
  void* out;
  int bf16;
  int64_t ld, stride;
  float keep, rate;
  float coef[3 * 64];
  int steps;
};

__host__ __device__ constexpr int small_ld(int nl) { return (nl + 63) / 64 * 64 + 8; }      // rows 16 bytes off a multiple of 128
__host__ __device__ constexpr int small_bytes(int nl) { return 2 * 2 * kSmall * (small_ld(nl) + 2 * kSmallLd); }

struct Halves { __half *hi, *lo; int ld; };

__device__ __forceinline__ void ld_matrix(uint32_t (&r)[4], const __half* p) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(smem_addr(p)) : "memory");
}
__device__ __forceinline__ void ld_matrix_trans(uint32_t (&r)[4], const __half* p) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(smem_addr(p)) : "memory");
}
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// acc = the warp's 16 x 16 entries, rows i0 .. and columns j0 .., of P Q^T (rows of both along the contraction index), or with
// kTrans of P Q (Q's rows are the contraction index).
template <bool kTrans>
__device__ __forceinline__ void small_product(const Halves& p, const Halves& q, int depth, int i0, int j0, float (&acc)[2][4]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[n][i] = 0.f;
  const int at_p = (i0 + (lane & 15)) * p.ld + (lane >> 4) * 8;
  const int at_q = kTrans ? (lane & 15) * q.ld + j0 + (lane >> 4) * 8 : (j0 + (lane & 7) + (lane >> 4) * 8) * q.ld + ((lane >> 3) & 1) * 8;
  const int step_q = kTrans ? 16 * q.ld : 16;
#pragma unroll 4
  for (int k = 0; k < depth; k += 16) {
    uint32_t ph[4], pl[4], qh[4], ql[4];
    ld_matrix(ph, p.hi + at_p + k);
    ld_matrix(pl, p.lo + at_p + k);
    const int iq = at_q + k / 16 * step_q;
    if (kTrans) {
      ld_matrix_trans(qh, q.hi + iq);
      ld_matrix_trans(ql, q.lo + iq);
    } else {
      ld_matrix(qh, q.hi + iq);
      ld_matrix(ql, q.lo + iq);
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      mma_16x8x16(acc[n], pl, qh[2 * n], qh[2 * n + 1]);
      mma_16x8x16(acc[n], ph, ql[2 * n], ql[2 * n + 1]);
      mma_16x8x16(acc[n], ph, qh[2 * n], qh[2 * n + 1]);
    }
  }
}
__device__ __forceinline__ void small_split(float a, float b, __half2& hi, __half2& lo) {
  hi = __floats2half2_rn(a, b);
  const float2 h = __half22float2(hi);
  lo = __floats2half2_rn(a - h.x, b - h.y);
}
// Entries (row, col) and (row, col + 1).
__device__ __forceinline__ void small_store(const Halves& m, int row, int col, float a, float b) {
  __half2 hi, lo;
  small_split(a, b, hi, lo);
  *(__half2*)(m.hi + row * m.ld + col) = hi;
  *(__half2*)(m.lo + row * m.ld + col) = lo;
}
__device__ __forceinline__ float2 small_load(const Halves& m, int row, int col) {
  const float2 h = __half22float2(*(const __half2*)(m.hi + row * m.ld + col)), l = __half22float2(*(const __half2*)(m.lo + row * m.ld + col));
  return make_float2(h.x + l.x, h.y + l.y);
}

__global__ void __launch_bounds__(kSmallThreads) k_orth_small(const __grid_constant__ Source s, const __grid_constant__ SmallOut to, int transpose) {
  extern __shared__ __align__(16) __half small_smem[];
  __shared__ double part[kSmallThreads / 32];
  const int z = blockIdx.x, t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int ns = transpose ? s.n : s.m, nl = transpose ? s.m : s.n, ld = small_ld(nl), count = s.m * s.n;
  const int chunks = (nl + 63) / 64, ks = (ns + 15) / 16 * 16, kl = (nl + 15) / 16 * 16;
  const Halves x = {small_smem, small_smem + kSmall * ld, ld};
  const Halves g = {x.lo + kSmall * ld, x.lo + kSmall * (ld + kSmallLd), kSmallLd};
  const Halves b = {g.lo + kSmall * kSmallLd, g.lo + 2 * kSmall * kSmallLd, kSmallLd};
  for (int i = t; i < kSmall * ld; i += kSmallThreads) *((uint32_t*)x.hi + i) = 0u;      // both halves
  launch_wait();
  launch_next();
  float u[kSmallKeep];
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < kSmallKeep; ++i) {
    const int k = t + i * kSmallThreads;
    u[i] = 0.f;
    if (k >= count) continue;
    const int r = k / s.n, c = k - r * s.n;
    u[i] = source_at(s, z * s.stride + r * s.ld + c);
    if (s.v) {
      float* v = s.v + z * s.v_stride + r * s.v_ld + c;
      const float nv = fmaf(s.mu, *v, u[i]);
      *v = nv;
      u[i] = update_of(s, u[i], nv);
    }
    sum += (double)u[i] * (double)u[i];
  }
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if (lane == 0) part[warp] = sum;
  __syncthreads();
  sum = 0.0;
  for (int i = 0; i < kSmallThreads / 32; ++i) sum += part[i];
  const float inv = sum == 0.0 ? 0.f : (float)((double)kSmallScale / (sqrt(sum) + (double)s.eps));
#pragma unroll
  for (int i = 0; i < kSmallKeep; ++i) {
    const int k = t + i * kSmallThreads;
    if (k >= count) continue;
    const int r = k / s.n, c = k - r * s.n, at = transpose ? c * ld + r : r * ld + c;
    const float v = u[i] * inv;
    const __half h = to_half(v);
    x.hi[at] = h;
    x.lo[at] = to_half(v - __half2float(h));
  }
  __syncthreads();
  const int i0 = (warp & 3) * 16, j0 = (warp >> 2) * 16;
  const int row = i0 + lane / 4, col = j0 + (lane & 3) * 2;      // of acc[n][0]: column + 8 n; acc[n][2]: row + 8
  float acc[2][4];
  for (int step = 0; step < to.steps; ++step) {
    const float ca = to.coef[3 * step] * kSmallScale, cb = to.coef[3 * step + 1], cc = to.coef[3 * step + 2] * (1.f / kSmallScale);
    small_product<false>(x, x, kl, i0, j0, acc);
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        small_store(g, row + 8 * h, col + 8 * n, acc[n][2 * h] * (1.f / kSmallScale), acc[n][2 * h + 1] * (1.f / kSmallScale));
    __syncthreads();
    small_product<false>(g, g, ks, i0, j0, acc);
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = row + 8 * h, c = col + 8 * n;
        const float2 a = small_load(g, r, c);
        small_store(b, r, c, cc * acc[n][2 * h] + cb * a.x + (r == c ? ca : 0.f), cc * acc[n][2 * h + 1] + cb * a.y + (r == c + 1 ? ca : 0.f));
      }
    __syncthreads();
    for (int k = 0; k < chunks; ++k) {
      small_product<true>(b, x, ks, i0, k * 64 + j0, acc);
      __syncthreads();      // these 64 columns of X have been read
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          small_store(x, row + 8 * h, k * 64 + col + 8 * n, acc[n][2 * h] * (1.f / kSmallScale), acc[n][2 * h + 1] * (1.f / kSmallScale));
    }
    __syncthreads();
  }
  for (int k = t; k < count; k += kSmallThreads) {
    const int r = k / s.n, c = k - r * s.n, from = transpose ? c * ld + r : r * ld + c;
    const float v = (__half2float(x.hi[from]) + __half2float(x.lo[from])) * (1.f / kSmallScale);
    const int64_t at = z * to.stride + r * to.ld + c;
    if (to.w) to.w[at] = to.keep * to.w[at] - to.rate * v;
    else if (to.bf16) ((__nv_bfloat16*)to.out)[at] = __float2bfloat16_rn(v);
    else ((float*)to.out)[at] = v;
  }
}

}  // namespace mat
}  // namespace rtopk
