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

// X = (u up) by.  One binary32 factor would be infinite for norms below 1e-37, which eps = 0 allows, and subnormal for norms above
// 3e39; up is 1 in between.
struct Factor {
  float up, by;
  __device__ __forceinline__ float operator()(float u) const { return u * up * by; }
};
__device__ __forceinline__ Factor factor_of(double sum_of_squares, float eps, float scale) {
  if (sum_of_squares == 0.0) return {1.f, 0.f};
  const double f = (double)scale / (sqrt(sum_of_squares) + (double)eps);
  const double up = f > 0x1p120 ? 0x1p64 : f < 0x1p-120 ? 0x1p-64 : 1.0;
  return {(float)up, (float)(f / up)};
}

// Sums of squares, in binary64 so that neither large nor small gradients leave the range; one partial sum per block, added
// up in a fixed order by the readers.  A warp takes 1024 neighbours of a row at a time, all loads under way before the first is
// used: bound by memory, four updates of 6000 x 1500 (432 MB) 44 us where part of them is still in L2.
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

// X, 64 x 64 elements of U per block, transposed when U is tall.  A thread writes eight neighbours of a row of X; four threads together give one partial sum of squares.  Bound by memory: four updates of 6000 x 1500 (504 MB) 69 us.
__global__ void __launch_bounds__(256)
k_split(const __grid_constant__ Source s, float* x, __half* h, int64_t ld, int64_t stride, float* row_sums, int slots, int64_t d_stride, int transpose) {
  __shared__ float tile[64][65];
  __shared__ Factor factor_s;
  const int z = blockIdx.z, c0 = blockIdx.x * 64, r0 = blockIdx.y * 64;
  launch_wait();
  launch_next();
  if (threadIdx.x < 32) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < s.parts; i += 32) sum += s.part[z * kNormBlocks + i];
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (threadIdx.x == 0) factor_s = factor_of(sum, s.eps, kXScale);
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
  const Factor scaled = factor_s;
  x += z * stride, h += z * stride, row_sums += (int64_t)z * slots * d_stride;
  const int ns = transpose ? s.n : s.m, nl = transpose ? s.m : s.n;
  const int a0 = transpose ? c0 : r0, b0 = transpose ? r0 : c0;      // of X: rows and columns
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int a = (threadIdx.x >> 3) + 32 * i, b = (threadIdx.x & 7) * 8;
    float u[8], sum = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      u[j] = scaled(transpose ? tile[b + j][a] : tile[a][b + j]);
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
// shared and tensor memory.  A chain of launches would spend its time starting them: at 64 x 64 a step's three products are 1.6
// million operations.  What bounds this kernel is the chain of fifteen dependent products, each of which goes from shared
// memory through the tensor core and tensor memory back to shared memory.  Every factor is the sum of two 16-bit numbers, high
// and low, and three of the four partial products are formed: 2^-21 of the result is lost, so that a matrix too small for
// errors to average out is as exact as a large one.
//
// A tile is 64 x 64 16-bit numbers in rows of 128 bytes, swizzled; X is a row of them.  The same bytes serve as a K-major
// operand (its rows along the contraction index) and as an MN-major one (its rows are the contraction index).  The tensor core's 128
// lanes reach 64 rows past a tile; what they make of those is not read.
//
// Measured: 64 x 64 17.7 us, 64 x 256 38 us (a chain of launches: 60 and 62).  One product takes about 2000 cycles: 740 for twelve
// matrix instructions, 190 to read tensor memory, 800 to split and store (half of the warps: lanes 64 to 127 hold nothing), 200 for
// the barrier.  mma.sync on the same halves takes 32 cycles an instruction and scheduler: 23 us at 64 x 64.
constexpr int kSmall = 64, kSmallLong = 256, kSmallThreads = 512;
constexpr int kSmallKeep = kSmall * kSmallLong / kSmallThreads;      // elements of U in a thread's registers
constexpr int kSmallBatch = 8;                                       // of them whose loads are under way together
constexpr float kSmallScale = 32.f;                                  // of X, its Gram matrix and the polynomial
constexpr int kTileBytes = kSmall * kDepthBytes;

struct SmallOut {
  float* w;                // update: the weights; null: out
  void* out;
  int bf16;
  int64_t ld, stride;
  float keep, rate;
  float coef[3 * 64];
  int steps;
  int test_giveup;         // tests only: every wait for a product counts as run out
};

__host__ __device__ constexpr int small_chunks(int nl) { return (nl + kSmall - 1) / kSmall; }
// X's, the Gram matrix's and the polynomial's tiles, high and low; the rows past the last one; alignment
__host__ __device__ constexpr int small_bytes(int nl) { return (2 * small_chunks(nl) + 4 + 1) * kTileBytes + 1024; }

// Byte of entry (row, col) of a tile.
__device__ __forceinline__ int tile_byte(int row, int col) { return row * kDepthBytes + (((col >> 3) ^ (row & 7)) << 4) + (col & 7) * 2; }

// Sixteen neighbours of a row of a tile, as high and low halves.
__device__ __forceinline__ void small_store(char* hi, char* lo, int row, int col, const float (&v)[16]) {
#pragma unroll
  for (int c = 0; c < 16; c += 8) {
    __half2 h[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      h[i] = __floats2half2_rn(v[c + 2 * i], v[c + 2 * i + 1]);
      const float2 f = __half22float2(h[i]);
      l[i] = __floats2half2_rn(v[c + 2 * i] - f.x, v[c + 2 * i + 1] - f.y);
    }
    const int at = tile_byte(row, col + c);
    *(uint4*)(hi + at) = *(uint4*)h;
    *(uint4*)(lo + at) = *(uint4*)l;
  }
}

// d (+)= P Q^T, or with kTrans P Q, of one pair of tiles with their low halves; by one whole warp.
template <bool kTrans>
__device__ __forceinline__ void small_product(uint32_t d, uint32_t p_hi, uint32_t p_lo, uint32_t q_hi, uint32_t q_lo, bool accumulate) {
  constexpr uint32_t kDesc = instr_desc(false, false, 128, kSmall, kTrans);
  constexpr int kStep = kTrans ? 2048 >> 4 : 2;
  const uint64_t ph = smem_desc(p_hi, 16), pl = smem_desc(p_lo, 16), qh = smem_desc(q_hi, kTileBytes), ql = smem_desc(q_lo, kTileBytes);
  if (elect_one()) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      tc_mma<false, false>(d, pl + k * 2, qh + k * kStep, kDesc, accumulate || k);
      tc_mma<false, false>(d, ph + k * 2, ql + k * kStep, kDesc, 1);
      tc_mma<false, false>(d, ph + k * 2, qh + k * kStep, kDesc, 1);
    }
  }
  __syncwarp();
}

__global__ void __launch_bounds__(kSmallThreads) k_orth_small(const __grid_constant__ Source s, const __grid_constant__ SmallOut to, int transpose, uint32_t* error) {
  extern __shared__ char small_smem[];
  __shared__ double part[kSmallThreads / 32];
  __shared__ __align__(8) uint64_t done, drain;
  __shared__ volatile uint32_t words[2];      // tensor-memory address, give-up word
  const int z = blockIdx.x, t = threadIdx.x, lane = t & 31, warp = __shfl_sync(0xFFFFFFFFu, t >> 5, 0);
  const int nl = transpose ? s.m : s.n;
  const int chunks = small_chunks(nl), bytes = chunks * kTileBytes;
  const uint32_t at_smem = smem_addr(small_smem), base = (at_smem + 1023u) & ~1023u;
  char* x_hi = small_smem + (base - at_smem);
  char *x_lo = x_hi + bytes, *g_hi = x_lo + bytes, *g_lo = g_hi + kTileBytes, *b_hi = g_lo + kTileBytes, *b_lo = b_hi + kTileBytes;
  const uint32_t x = base, g = base + 2 * bytes, b = g + 2 * kTileBytes, bar = smem_addr(&done);
  const uint32_t tmem_cols = chunks <= 1 ? 64 : chunks <= 2 ? 128 : 256;
  const GiveUp give{words + 1, error};
  if (t == 0) {
    bar_init(bar, 1);
    bar_init(smem_addr(&drain), 1);
    words[1] = 0u;
    bar_init_fence();
  }
  if (warp == 0) tmem_alloc<false>(smem_addr((const void*)words), tmem_cols);
  for (int i = t * 16; i < 2 * bytes; i += kSmallThreads * 16) *(uint4*)(x_hi + i) = make_uint4(0u, 0u, 0u, 0u);
  launch_wait();
  launch_next();
  // Element i of a thread: entry t + 512 i of U with its rows padded to a power of two; entries outside U read its first one.
  const int shift = s.n <= 32 ? 5 : 32 - __clz(s.n - 1), turns = ((s.m << shift) + kSmallThreads - 1) / kSmallThreads;
  auto entry = [&](int i, int& r, int& c) {
    const int k = t + i * kSmallThreads;
    r = k >> shift, c = k & ((1 << shift) - 1);
    return r < s.m && c < s.n;
  };
  float u[kSmallKeep];
  double sum = 0.0;
#pragma unroll
  for (int i0 = 0; i0 < kSmallKeep; i0 += kSmallBatch) {
    if (i0 >= turns) break;
    float v[kSmallBatch];
#pragma unroll
    for (int i = 0; i < kSmallBatch; ++i) {
      int r, c;
      const bool in = entry(i0 + i, r, c);
      u[i0 + i] = source_at(s, z * s.stride + (in ? r * s.ld + c : 0));
      if (s.v) v[i] = s.v[z * s.v_stride + (in ? r * s.v_ld + c : 0)];
    }
#pragma unroll
    for (int i = 0; i < kSmallBatch; ++i) {
      int r, c;
      const bool in = entry(i0 + i, r, c);
      float& e = u[i0 + i];
      if (s.v) {
        const float nv = fmaf(s.mu, v[i], e);
        if (in) s.v[z * s.v_stride + r * s.v_ld + c] = nv;
        e = update_of(s, e, nv);
      }
      if (in) sum += (double)e * (double)e;
    }
  }
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if (lane == 0) part[warp] = sum;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = words[0];
  sum = 0.0;
  for (int i = 0; i < kSmallThreads / 32; ++i) sum += part[i];
  const Factor scaled = factor_of(sum, s.eps, kSmallScale);
#pragma unroll
  for (int i = 0; i < kSmallKeep; ++i) {
    if (i >= turns) break;
    int r, c;
    if (!entry(i, r, c)) continue;
    const int row = transpose ? c : r, col = transpose ? r : c, at = col / kSmall * kTileBytes + tile_byte(row, col & (kSmall - 1));
    const float v = scaled(u[i]);
    const __half h = to_half(v);
    *(__half*)(x_hi + at) = h;
    *(__half*)(x_lo + at) = to_half(v - __half2float(h));
  }
  smem_publish();
  __syncthreads();
  // tensor memory's lanes 0 .. 63 belong to the warps 0 and 1 of every four: eight warps at work, 32 rows x 16 columns each
  const bool works = (warp & 3) < 2;
  const int row = (warp & 3) * 32 + lane, col = (warp >> 2) * 16;
  const uint32_t from = tmem + ((uint32_t)((warp & 3) * 32) << 16) + col;
  uint32_t phase = 0;
  bool failed = false;
  // ends a product: its results, once it is done
  auto result = [&](int c0, float (&v)[16], float scale) {
    uint32_t acc[16];
    tmem_load16(from + c0, acc);
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(acc[i]) * scale;
  };
  auto wait = [&]() {
    if (works) {
      if (!__all_sync(0xFFFFFFFFu, to.test_giveup ? give_up(give) : bar_wait(bar, phase, give))) failed = true;
      tc_fence_after();
    }
    phase ^= 1;
  };
  auto publish = [&]() {
    tc_fence_before();
    smem_publish();
    failed = __syncthreads_or(failed) != 0;
    tc_fence_after();
  };
  for (int step = 0; step < to.steps; ++step) {
    const float ca = to.coef[3 * step] * kSmallScale, cb = to.coef[3 * step + 1], cc = to.coef[3 * step + 2] * (1.f / kSmallScale);
    float gram[16], v[16];
    if (warp == 0) {
      for (int c = 0; c < chunks; ++c) {
        const uint32_t at = x + c * kTileBytes;
        small_product<false>(tmem, at, at + bytes, at, at + bytes, c > 0);
      }
      if (elect_one()) tc_commit<false>(bar);
      __syncwarp();
    }
    wait();
    if (works) {
      result(0, gram, 1.f / kSmallScale);
      small_store(g_hi, g_lo, row, col, gram);
    }
    publish();
    if (failed) break;
    if (warp == 0) {
      small_product<false>(tmem, g, g + kTileBytes, g, g + kTileBytes, false);
      if (elect_one()) tc_commit<false>(bar);
      __syncwarp();
    }
    wait();
    if (works) {
      result(0, v, cc);
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] += cb * gram[i] + (row == col + i ? ca : 0.f);
      small_store(b_hi, b_lo, row, col, v);
    }
    publish();
    if (failed) break;
    if (warp == 0) {
      for (int c = 0; c < chunks; ++c) small_product<true>(tmem + c * kSmall, b, b + kTileBytes, x + c * kTileBytes, x + bytes + c * kTileBytes, false);
      if (elect_one()) tc_commit<false>(bar);
      __syncwarp();
    }
    wait();
    if (works)
      for (int c = 0; c < chunks; ++c) {
        result(c * kSmall, v, 1.f / kSmallScale);
        small_store(x_hi + c * kTileBytes, x_lo + c * kTileBytes, row, col, v);
      }
    publish();
    if (failed) break;
  }
  if (failed) {
    if (warp == 0 && elect_one()) {
      tc_commit<false>(smem_addr(&drain));
      bar_drain(smem_addr(&drain), 0, now_ns());
    }
    __syncthreads();
  }
  if (warp == 0) tmem_free<false>(tmem, tmem_cols);
  if (failed) return;
#pragma unroll 1
  for (int i0 = 0; i0 < turns; i0 += kSmallBatch) {
    float w[kSmallBatch];
#pragma unroll
    for (int i = 0; i < kSmallBatch; ++i) {
      int r, c;
      const bool in = entry(i0 + i, r, c);
      if (to.w) w[i] = to.w[z * to.stride + (in ? r * to.ld + c : 0)];
    }
#pragma unroll
    for (int i = 0; i < kSmallBatch; ++i) {
      int r, c;
      if (!entry(i0 + i, r, c)) continue;
      const int row = transpose ? c : r, col = transpose ? r : c, from_x = col / kSmall * kTileBytes + tile_byte(row, col & (kSmall - 1));
      const float v = (__half2float(*(const __half*)(x_hi + from_x)) + __half2float(*(const __half*)(x_lo + from_x))) * (1.f / kSmallScale);
      const int64_t at = z * to.stride + r * to.ld + c;
      if (to.w) to.w[at] = to.keep * w[i] - to.rate * v;
      else if (to.bf16) ((__nv_bfloat16*)to.out)[at] = __float2bfloat16_rn(v);
      else ((float*)to.out)[at] = v;
    }
  }
}

// The shorter side at most 128, the longer at most 2048: one cluster of up to eight blocks per matrix, 256 columns of X a block.  A
// launch for each product would take 5 to 7 us here, most of it for starting and for the first bytes to arrive; in the
// cluster X never leaves the SMs (in 32 bits in registers, in 16 bits as the products' operand in shared memory), each block
// forms the polynomial for itself, and only the blocks' shares of the Gram matrix meet, through distributed shared memory: each
// block adds up its part of the entries in the blocks' order and hands the sum to all.  The arithmetic is that of the
// product kernel: 16-bit operands, X and the diagonals in 32 bits.
//
// Measured, against a chain of launches, us: 128 x 128 29 / 61, 128 x 256 40 / 63, 128 x 1000 68 / 71, 128 x 2048 76 / 80, thirty of
// 128 x 1000 73 / 122.  A step is about 5800 cycles in one block; in a cluster 18700, 9200 of them the exchange of 96 KB a
// block through distributed shared memory at about 16 bytes a cycle.  512 threads leave 128 registers for each; 124 bytes a thread spill.
constexpr int kMid = 128, kMidThreads = 512, kMidChunks = 4, kMidCluster = 8, kMidLong = kMidCluster * kMidChunks * kSmall;
constexpr int kMidTile = kMid * kDepthBytes;                          // 128 rows of 64 16-bit numbers
constexpr int kMidPart = kMid * kMid * 4, kMidPitch = kSmall + 1;
constexpr int kMidBytes = (kMidChunks + 2 + 2) * kMidTile + kMidPart + 1024;      // X, the Gram matrix, the polynomial, the block's share

__global__ void __launch_bounds__(kMidThreads, 1) k_orth_cluster(const __grid_constant__ Source s, const __grid_constant__ SmallOut to, int transpose, int chunks, uint32_t* error) {
  extern __shared__ char mid_smem[];
  __shared__ double warp_sum[kMidThreads / 32], norms[kMidCluster];
  __shared__ __align__(16) float gram_d[kMid];
  __shared__ float poly_d[kMid], row_part[4][kMid], row_sums[kMidCluster][kMid];
  __shared__ __align__(8) uint64_t done, drain;
  __shared__ volatile uint32_t words[2];      // tensor-memory address, give-up word
  uint32_t blocks;
  asm volatile("mov.u32 %0, %cluster_nctaid.x;" : "=r"(blocks));
  const uint32_t rank = rank_in_cluster();
  const int z = blockIdx.x / blocks, t = threadIdx.x, lane = t & 31, warp = __shfl_sync(0xFFFFFFFFu, t >> 5, 0);
  const int ns = transpose ? s.n : s.m, nl = transpose ? s.m : s.n;
  const uint32_t at_smem = smem_addr(mid_smem), x_at = (at_smem + 1023u) & ~1023u;
  char* x_tile = mid_smem + (x_at - at_smem);
  char *g_tile = x_tile + kMidChunks * kMidTile, *b_tile = g_tile + 2 * kMidTile;
  float4* share = (float4*)(b_tile + 2 * kMidTile);                   // [column / 4][row]
  const uint32_t g_at = x_at + kMidChunks * kMidTile, b_at = g_at + 2 * kMidTile, share_at = b_at + 2 * kMidTile, bar = smem_addr(&done);
  const GiveUp give{words + 1, error};
  if (t == 0) {
    bar_init(bar, 1);
    bar_init(smem_addr(&drain), 1);
    words[1] = 0u;
    bar_init_fence();
  }
  if (warp == 0) tmem_alloc<false>(smem_addr((const void*)words), 512);
  launch_wait();
  launch_next();
  // A thread's part of X: its lane's row, 16 columns of each of the block's chunks.  It comes by way of the tiles' room, where
  // a chunk takes 128 rows of 65 numbers, so that neighbours of a row of U are read together.
  const int quarter = warp & 3, group = warp >> 2, row = quarter * 32 + lane;
  const int col0 = rank * chunks * kSmall;
  float* stage = (float*)x_tile;
  auto entry = [&](int c, int i, int& r, int& k) {      // entry i of a thread of chunk c: row and column of X; whether it exists
    const int e = t + i * kMidThreads;
    r = transpose ? e & (kMid - 1) : e >> 6, k = transpose ? e >> 7 : e & (kSmall - 1);
    return r < ns && col0 + c * kSmall + k < nl;
  };
  auto offset = [&](int c, int r, int k, int64_t ld) { return transpose ? (int64_t)(col0 + c * kSmall + k) * ld + r : r * ld + col0 + c * kSmall + k; };
  double sum = 0.0;
#pragma unroll 1
  for (int c = 0; c < chunks; ++c) {
    float u[16], v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      int r, k;
      const bool in = entry(c, i, r, k);
      u[i] = source_at(s, z * s.stride + (in ? offset(c, r, k, s.ld) : 0));
      if (s.v) v[i] = s.v[z * s.v_stride + (in ? offset(c, r, k, s.v_ld) : 0)];
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      int r, k;
      const bool in = entry(c, i, r, k);
      if (s.v) {
        const float nv = fmaf(s.mu, v[i], u[i]);
        if (in) s.v[z * s.v_stride + offset(c, r, k, s.v_ld)] = nv;
        u[i] = update_of(s, u[i], nv);
      }
      if (!in) u[i] = 0.f;
      sum += (double)u[i] * (double)u[i];
      stage[(c * kMid + r) * kMidPitch + k] = u[i];
    }
  }
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if (lane == 0) warp_sum[warp] = sum;
  tc_fence_before();
  cluster_sync();      // every block of the cluster has started
  tc_fence_after();
  const uint32_t tmem = words[0];
  if (t < (int)blocks) {
    sum = 0.0;
    for (int i = 0; i < kMidThreads / 32; ++i) sum += warp_sum[i];
    cluster_store(at_rank(smem_addr(norms + rank), t), sum);
  }
  cluster_sync();
  sum = 0.0;
  for (uint32_t i = 0; i < blocks; ++i) sum += norms[i];
  const Factor scaled = factor_of(sum, s.eps, kXScale);
  float x[kMidChunks][16];
#pragma unroll
  for (int c = 0; c < kMidChunks; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) x[c][i] = c < chunks ? scaled(stage[(c * kMid + row) * kMidPitch + group * 16 + i]) : 0.f;
  __syncthreads();

  // Sixteen neighbours of a row of a tile.
  auto store16 = [&](char* tile, int col, const float* v) {
    store_half8((__half*)(tile + tile_byte(row, col)), v);
    store_half8((__half*)(tile + tile_byte(row, col + 8)), v + 8);
  };
  auto publish = [&]() {
    tc_fence_before();
    smem_publish();
    __syncthreads();
    tc_fence_after();
  };
  uint32_t phase = 0;
  auto wait = [&]() {      // a block that gives up goes on, so that the others' barriers are met; its results mean nothing
    __syncwarp();
    if (to.test_giveup) give_up(give);
    bar_wait(bar, phase, give);
    phase ^= 1;
    __syncwarp();
    tc_fence_after();
  };
  const uint32_t from = tmem + ((uint32_t)(quarter * 32) << 16);
  const int own = 32 / blocks;      // groups of four columns of the Gram matrix that this block adds up
  for (int step = 0; step < to.steps; ++step) {
    const float ca = to.coef[3 * step], cb = to.coef[3 * step + 1], cc = to.coef[3 * step + 2];
    // X as the products' operand, and the squares of its rows
    float squares = 0.f;
#pragma unroll
    for (int c = 0; c < kMidChunks; ++c) {
      if (c >= chunks) break;
#pragma unroll
      for (int i = 0; i < 16; ++i) squares = fmaf(x[c][i], x[c][i], squares);
      store16(x_tile + c * kMidTile, group * 16, x[c]);
    }
    row_part[group][row] = squares;
    publish();
    // the Gram matrix
    if (warp == 0) {
      constexpr uint32_t kDesc = instr_desc(false, false, kMid, kMid);
      for (int c = 0; c < chunks; ++c) {
        const uint64_t d = smem_desc(x_at + c * kMidTile, 16);
        if (elect_one())
#pragma unroll
          for (int k = 0; k < 4; ++k) tc_mma<false, false>(tmem, d + k * 2, d + k * 2, kDesc, c > 0 || k);
        __syncwarp();
      }
      if (elect_one()) tc_commit<false>(bar);
      __syncwarp();
    }
    if (blocks == 1) {
      if (t < kMid) gram_d[t] = ((row_part[0][t] + row_part[1][t]) + (row_part[2][t] + row_part[3][t])) * (1.f / kAScale);
      wait();
      uint32_t acc[32];
      tmem_load32(from + group * 32, acc);
      float v[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = group == quarter && lane == i ? 0.f : __uint_as_float(acc[i]);      // the diagonal is kept apart
      char* tile = g_tile + group * 32 / kSmall * kMidTile;
      store16(tile, group * 32 % kSmall, v);
      store16(tile, group * 32 % kSmall + 16, v + 16);
      publish();
    } else {
      if (t >= 32 && t < 32 + (int)(blocks * 16)) {      // eight rows' sums to one block each
        const uint32_t peer = (t - 32) >> 4;
        for (int r = ((t - 32) & 15) * 8, e = r + 8; r < e; ++r)
          cluster_store(at_rank(smem_addr(&row_sums[rank][r]), peer), (row_part[0][r] + row_part[1][r]) + (row_part[2][r] + row_part[3][r]));
      }
      wait();
      {
        uint32_t acc[32];
        tmem_load32(from + group * 32, acc);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          share[(group * 8 + i) * kMid + row] =
              make_float4(__uint_as_float(acc[4 * i]), __uint_as_float(acc[4 * i + 1]), __uint_as_float(acc[4 * i + 2]), __uint_as_float(acc[4 * i + 3]));
      }
      tc_fence_before();
      cluster_sync();
      for (int i = t; i < own * kMid; i += kMidThreads) {
        const int col4 = rank * own + i / kMid, r = i % kMid;
        float4 w[kMidCluster], v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (uint32_t p = 0; p < kMidCluster; ++p)
          if (p < blocks) w[p] = cluster_load4(at_rank(share_at + (col4 * kMid + r) * 16, p));
#pragma unroll
        for (uint32_t p = 0; p < kMidCluster; ++p)
          if (p < blocks) v.x += w[p].x, v.y += w[p].y, v.z += w[p].z, v.w += w[p].w;
        const int off = r - col4 * 4;      // the diagonal is kept apart
        __half2 h[2] = {__floats2half2_rn(off == 0 ? 0.f : v.x, off == 1 ? 0.f : v.y), __floats2half2_rn(off == 2 ? 0.f : v.z, off == 3 ? 0.f : v.w)};
        const uint32_t at = g_at + (col4 / 16) * kMidTile + tile_byte(r, col4 % 16 * 4);
#pragma unroll
        for (uint32_t p = 0; p < kMidCluster; ++p)
          if (p < blocks) cluster_store(at_rank(at, p), *(uint2*)h);
      }
      if (t < kMid) {
        float d = 0.f;
        for (uint32_t p = 0; p < blocks; ++p) d += row_sums[p][t];
        gram_d[t] = d * (1.f / kAScale);
      }
      cluster_publish();
      cluster_sync();
      cluster_publish();
      tc_fence_after();
    }
    // the polynomial
    if (warp == 0) {
      constexpr uint32_t kDesc = instr_desc(false, false, kMid, kMid);
      const uint64_t d = smem_desc(g_at, 16);
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint64_t at = d + k / 4 * (kMidTile >> 4) + k % 4 * 2;
          tc_mma<false, false>(tmem, at, at, kDesc, k > 0);
        }
        tc_commit<false>(bar);
      }
      __syncwarp();
    }
    wait();
    {
      uint32_t acc[32];
      tmem_load32(from + group * 32, acc);
      const float dl = gram_d[row], base = cb + cc * dl, scale = cc * (1.f / kAScale);
      if (group == quarter) {      // the warps whose columns hold their rows' diagonal
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          q = lane == i ? __uint_as_float(acc[i]) : q;
          acc[i] = lane == i ? 0u : acc[i];      // the Gram matrix holds 0 there too
        }
        poly_d[row] = ca + cb * dl + cc * (dl * dl + q * (1.f / (kAScale * kAScale)));
      }
#pragma unroll
      for (int c = 0; c < 32; c += 8) {
        const int col = group * 32 + c, at = col / kSmall * kMidTile + tile_byte(row, col % kSmall);
        const uint4 w = *(const uint4*)(g_tile + at);
        const __half2* g = (const __half2*)&w;
        const float4 d0 = *(const float4*)(gram_d + col), d1 = *(const float4*)(gram_d + col + 4);
        const float dc[8] = {d0.x, d0.y, d0.z, d0.w, d1.x, d1.y, d1.z, d1.w};
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const float2 o = __half22float2(g[i / 2]);
          v[i] = fmaf(scale, __uint_as_float(acc[c + i]), fmaf(cc, dc[i], base) * o.x);
          v[i + 1] = fmaf(scale, __uint_as_float(acc[c + i + 1]), fmaf(cc, dc[i + 1], base) * o.y);
        }
        store_half8((__half*)(b_tile + at), v);
      }
    }
    publish();
    // X <- (that) X
    if (warp == 0) {
      const uint32_t desc = instr_desc(false, false, kMid, chunks * kSmall, true);
      const uint64_t dp = smem_desc(b_at, 16), dq = smem_desc(x_at, kMidTile);
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < 8; ++k) tc_mma<false, false>(tmem + kMid, dp + k / 4 * (kMidTile >> 4) + k % 4 * 2, dq + k * (2048 >> 4), desc, k > 0);
        tc_commit<false>(bar);
      }
      __syncwarp();
    }
    wait();
    const float d = poly_d[row];
#pragma unroll
    for (int c = 0; c < kMidChunks; ++c) {
      if (c >= chunks) break;
      uint32_t acc[16];
      tmem_load16(from + kMid + c * kSmall + group * 16, acc);
#pragma unroll
      for (int i = 0; i < 16; ++i) x[c][i] = d * x[c][i] + __uint_as_float(acc[i]) * (1.f / kAScale);
    }
  }
  __syncwarp();
  if (words[1] && warp == 0 && elect_one()) {
    tc_commit<false>(smem_addr(&drain));
    bar_drain(smem_addr(&drain), 0, now_ns());
  }
  tc_fence_before();
  cluster_sync();
  tc_fence_after();
  if (warp == 0) tmem_free<false>(tmem, 512);
#pragma unroll
  for (int c = 0; c < kMidChunks; ++c)
    if (c < chunks)
#pragma unroll
      for (int i = 0; i < 16; ++i) stage[(c * kMid + row) * kMidPitch + group * 16 + i] = x[c][i] * (1.f / kXScale);
  __syncthreads();
#pragma unroll 1
  for (int c = 0; c < chunks; ++c) {
    float w[16];
    if (to.w)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        int r, k;
        const bool in = entry(c, i, r, k);
        w[i] = to.w[z * to.stride + (in ? offset(c, r, k, to.ld) : 0)];
      }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      int r, k;
      if (!entry(c, i, r, k)) continue;
      const float v = stage[(c * kMid + r) * kMidPitch + k];
      const int64_t at = z * to.stride + offset(c, r, k, to.ld);
      if (to.w) to.w[at] = to.keep * w[i] - to.rate * v;
      else if (to.bf16) ((__nv_bfloat16*)to.out)[at] = __float2bfloat16_rn(v);
      else ((float*)to.out)[at] = v;
    }
  }
}

}  // namespace mat
}  // namespace rtopk
