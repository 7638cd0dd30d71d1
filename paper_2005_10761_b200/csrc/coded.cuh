// 8-bit codes with one binary32 scale for each row or column, and what makes them.
//
//   s = max |v| / 127,   q = rint(v / s) clamped to +-127      (both quotients rounded to binary32)
//
// over a row (one token, one output channel) or a column (one channel over the tokens).  An all-zero row has s = 0 and
// q = 0; a row with an infinity or a NaN has s = NaN and q = 0, so that everything it takes part in is NaN.
#pragma once

#include <cuda_bf16.h>

#include "tensorcore.cuh"

namespace rtopk {
namespace mat {

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }

// |v| as a bit pattern: ordered like the magnitudes, a NaN above everything, so that maxima of it are exact and
// independent of their order.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

__device__ __forceinline__ float code_scale(uint32_t max_magnitude) {
  if (max_magnitude >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  return __fdiv_rn(__uint_as_float(max_magnitude), 127.f);
}
// rint(v / s), the quotient formed.
__device__ __forceinline__ int code_exactly(float v, float s) { return max(-127, min(127, __float2int_rn(__fdiv_rn(v, s)))); }

// Codes without a division: adding 1.5 * 2^23 to v * r, r the reciprocal of s, rounds the exact product to a whole number and
// leaves it in the low byte of the sum.  The product is within 2^-23 of the quotient, 2e-5 at 127, so both round to the same
// code unless the product lies that near to the middle between two: `off` collects how far the products are from their codes,
// and where that comes to 0.4999 the quotients are formed after all.
constexpr float kToByte = 12582912.f;
__device__ __forceinline__ uint32_t code_byte(float v, float r, float& off) {
  const float t = fmaf(v, r, kToByte);
  off = fmaxf(off, fabsf(fmaf(v, r, kToByte - t)));
  return __float_as_uint(t);
}
__device__ __forceinline__ uint32_t pack_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
// The reciprocal for code_byte().  All codes are 0 without a positive scale (s = 1 then, r = 0); scales near the subnormal
// range have no usable reciprocal: infinity, which makes `off` NaN or infinite.
__device__ __forceinline__ float code_reciprocal(float& s) {
  if (!(s > 0.f)) { s = 1.f; return 0.f; }
  return s < 1e-36f ? __uint_as_float(0x7F800000u) : __fdiv_rn(1.f, s);
}
// Four codes in a word.  With r = 0 the values may be anything, infinities and NaN too.
__device__ __forceinline__ uint32_t code4(float a, float b, float c, float d, float s, float r) {
  if (r == 0.f) return 0u;
  float off = 0.f;
  const uint32_t w = pack_bytes(code_byte(a, r, off), code_byte(b, r, off), code_byte(c, r, off), code_byte(d, r, off));
  if (off < 0.4999f && r < 1e37f) return w;
  return pack_bytes(code_exactly(a, s), code_exactly(b, s), code_exactly(c, s), code_exactly(d, s));
}

// Eight neighbours of a row; those past the end are zero.  `vec`: the row allows 16-byte loads.
__device__ __forceinline__ void load8(const float* p, int left, bool vec, float (&v)[8]) {
  if (vec && left >= 8) {
    const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : 0.f;
  }
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, int left, bool vec, float (&v)[8]) {
  if (vec && left >= 8) {
    const uint4 a = *(const uint4*)p;
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? widen(p[i]) : 0.f;
  }
}
__device__ __forceinline__ void times8(const float* mul, int left, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < left) v[i] *= mul[i];
}
__device__ __forceinline__ void code8(const float (&v)[8], int left, float s, float r, int8_t* out) {
  const uint32_t w[2] = {code4(v[0], v[1], v[2], v[3], s, r), code4(v[4], v[5], v[6], v[7], s, r)};
  if (left >= 8) {
    *(uint2*)out = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) out[i] = (int8_t)(w[i >> 2] >> (8 * (i & 3)));
  }
}

// Codes along the rows; kWarps warps per row.  `mul` (may be null) multiplies column c first.  Rows of up to
// kWarps * 1024 elements are read once and kept in registers, longer ones are read again for their codes.
template <class T, int kWarps>
__global__ void __launch_bounds__(256) k_code_rows(const T* src, int64_t ld, int rows, int cols, int vec, const float* mul, int8_t* codes, int64_t ld_codes, float* scales) {
  constexpr int kKeep = 4, kSpan = kWarps * 32 * 8;
  __shared__ uint32_t part[8];
  const int group = threadIdx.x / (32 * kWarps), t = threadIdx.x % (32 * kWarps);
  const int row = blockIdx.x * (8 / kWarps) + group;
  const bool in = row < rows;
  launch_wait();
  launch_next();
  const T* p = src + (int64_t)(in ? row : 0) * ld;
  float v[kKeep][8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kKeep; ++i) {
    const int c = i * kSpan + t * 8;
    if (c < cols) load8(p + c, cols - c, vec, v[i]);
  }
#pragma unroll
  for (int i = 0; i < kKeep; ++i) {
    const int c = i * kSpan + t * 8;
    if (c >= cols) continue;
    if (mul) times8(mul + c, cols - c, v[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, magnitude(v[i][j]));
  }
  for (int c = kKeep * kSpan + t * 8; c < cols; c += kSpan) {
    float u[8];
    load8(p + c, cols - c, vec, u);
    if (mul) times8(mul + c, cols - c, u);
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, magnitude(u[j]));
  }
  m = __reduce_max_sync(0xFFFFFFFFu, m);
  if (kWarps > 1) {
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
    __syncthreads();
    m = part[group * kWarps + (threadIdx.x & (kWarps - 1))];
    m = __reduce_max_sync(0xFFFFFFFFu, m);
  }
  if (!in) return;
  float s = code_scale(m);
  if (t == 0) scales[row] = s;
  const float r = code_reciprocal(s);
  int8_t* out = codes + row * ld_codes;
#pragma unroll
  for (int i = 0; i < kKeep; ++i) {
    const int c = i * kSpan + t * 8;
    if (c < cols) code8(v[i], cols - c, s, r, out + c);
  }
  for (int c = kKeep * kSpan + t * 8; c < cols; c += kSpan) {
    float u[8];
    load8(p + c, cols - c, vec, u);
    if (mul) times8(mul + c, cols - c, u);
    code8(u, cols - c, s, r, out + c);
  }
}

// Largest magnitude of every column (max_bits zeroed before): 256 columns per block, eight threads deep.
template <class T>
__global__ void __launch_bounds__(256) k_col_max(const T* src, int64_t ld, int rows, int cols, int vec, int rows_per_block, uint32_t* max_bits) {
  __shared__ uint32_t part[8][256];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
  const int c = blockIdx.x * 256 + x * 8;
  const int r0 = blockIdx.y * rows_per_block, r1 = min(rows, r0 + rows_per_block);
  launch_wait();
  launch_next();
  uint32_t m[8] = {};
  if (c < cols) {
#pragma unroll 8
    for (int r = r0 + y; r < r1; r += 8) {
      float v[8];
      load8(src + r * ld + c, cols - c, vec, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) m[i] = max(m[i], magnitude(v[i]));
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) part[y][i * 32 + x] = m[i];
  __syncthreads();
  uint32_t best = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) best = max(best, part[i][threadIdx.x]);
  const int col = blockIdx.x * 256 + x * 8 + y;     // entry y * 32 + x
  if (col < cols && best) atomicMax(max_bits + col, best);
}

// Codes for each column, written transposed: codes[c][r], scales[c].  128 rows x 64 columns per block; four codes of a
// column are one word, so that a row of the result leaves in 128-byte pieces.
template <class T>
__global__ void __launch_bounds__(256)
k_code_cols(const T* src, int64_t ld, int rows, int cols, int vec, const uint32_t* max_bits, int8_t* codes, int64_t ld_codes, float* scales) {
  __shared__ uint32_t tile[64][33];
  __shared__ float2 scale[64];
  const int c0 = blockIdx.x * 64, r0 = blockIdx.y * 128;
  const int cg = (threadIdx.x & 7) * 8, rg = threadIdx.x >> 3;
  launch_wait();
  launch_next();
  const int left = cols - c0 - cg;
  float v[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = r0 + rg * 4 + i;
    load8(src + (int64_t)min(r, rows - 1) * ld + c0 + cg, r < rows ? left : 0, vec, v[i]);
  }
  if (threadIdx.x < 64 && c0 + threadIdx.x < cols) {
    float s = code_scale(max_bits[c0 + threadIdx.x]);
    if (blockIdx.y == 0) scales[c0 + threadIdx.x] = s;
    const float r = code_reciprocal(s);
    scale[threadIdx.x] = make_float2(s, r);
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < left) {
      const float2 q = scale[cg + j];
      tile[cg + j][rg] = code4(v[0][j], v[1][j], v[2][j], v[3][j], q.x, q.y);
    }
  __syncthreads();
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
  const int n = min(4, rows - r0 - x * 4);
  for (int c = y; c < 64; c += 8) {
    if (c0 + c >= cols || n <= 0) continue;
    int8_t* out = codes + (int64_t)(c0 + c) * ld_codes + r0 + x * 4;
    const uint32_t w = tile[c][x];
    if (n == 4) *(uint32_t*)out = w;
    else
      for (int i = 0; i < n; ++i) out[i] = (int8_t)(w >> (8 * i));
  }
}

// codes_t[c][r] = codes[r][c].
__global__ void __launch_bounds__(256) k_codes_transpose(const int8_t* codes, int64_t ld, int rows, int cols, int8_t* out, int64_t ld_out) {
  __shared__ int8_t tile[64][65];
  const int c0 = blockIdx.x * 64, r0 = blockIdx.y * 64;
  launch_wait();
  launch_next();
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
  for (int r = y; r < 64; r += 4)
    if (r0 + r < rows && c0 + x < cols) tile[x][r] = codes[(int64_t)(r0 + r) * ld + c0 + x];
  __syncthreads();
  for (int c = y; c < 64; c += 4)
    if (c0 + c < cols && r0 + x < rows) out[(int64_t)(c0 + c) * ld_out + r0 + x] = tile[c][x];
}

// A linear layer for a few tokens: reading the codes of W once is all the work, so one launch does everything.  Each block
// codes the tokens for itself (they are small, and come from L2), then each warp takes two output channels at a time: 16 codes
// of W a thread, four-way integer dot products with the tokens' codes in shared memory.
constexpr int kFewThreads = 256;
constexpr int kFewBytes = 48 * 1024;       // codes of all tokens in shared memory, at most
__host__ __device__ constexpr int few_row(int n_in) { return (n_in + 511) / 512 * 512; }

template <class T, int kTokens>
__global__ void __launch_bounds__(kFewThreads)
k_product_few(const T* x, int64_t ld_x, int vec, const int8_t* codes, int64_t ld_codes, const float* scales, int tokens, int n_out, int n_in, T* out, int64_t ld_out) {
  extern __shared__ __align__(16) char few_smem[];
  __shared__ uint32_t part[8][kTokens];
  __shared__ float token_scale[kTokens];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = few_row(n_in);
  launch_wait();
  launch_next();
  uint32_t m[kTokens] = {};
  for (int c = threadIdx.x * 8; c < n_in; c += kFewThreads * 8)
#pragma unroll
    for (int t = 0; t < kTokens; ++t) {
      float v[8];
      load8(x + min(t, tokens - 1) * ld_x + c, n_in - c, vec, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) m[t] = max(m[t], magnitude(v[i]));
    }
#pragma unroll
  for (int t = 0; t < kTokens; ++t) {
    m[t] = __reduce_max_sync(0xFFFFFFFFu, m[t]);
    if (lane == 0) part[warp][t] = m[t];
  }
  __syncthreads();
  float s[kTokens], r[kTokens];
#pragma unroll
  for (int t = 0; t < kTokens; ++t) {
    uint32_t best = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) best = max(best, part[i][t]);
    s[t] = code_scale(best);
    if (threadIdx.x == 0) token_scale[t] = s[t];
    r[t] = code_reciprocal(s[t]);
  }
  for (int c = threadIdx.x * 8; c < row; c += kFewThreads * 8)
#pragma unroll
    for (int t = 0; t < kTokens; ++t) {
      float v[8];
      load8(x + min(t, tokens - 1) * ld_x + min(c, n_in - 1), max(n_in - c, 0), vec, v);
      *(uint2*)(few_smem + t * row + c) = make_uint2(code4(v[0], v[1], v[2], v[3], s[t], r[t]), code4(v[4], v[5], v[6], v[7], s[t], r[t]));
    }
  __syncthreads();
  const int pairs = (n_out + 1) / 2;
  for (int k = blockIdx.x * 8 + warp; k < pairs; k += gridDim.x * 8) {
    const int n0 = 2 * k, n1 = min(n0 + 1, n_out - 1);
    const int8_t *w0 = codes + n0 * ld_codes, *w1 = codes + n1 * ld_codes;
    int acc[2][kTokens] = {};
    // past the end of a row the tokens' codes are zero, so that the last 16 codes read there count for nothing
#pragma unroll 4
    for (int c = lane * 16; c < n_in; c += 512) {
      const int4 a = __ldg((const int4*)(w0 + c)), b = __ldg((const int4*)(w1 + c));
#pragma unroll
      for (int t = 0; t < kTokens; ++t) {
        const int4 q = *(const int4*)(few_smem + t * row + c);
        acc[0][t] = __dp4a(a.x, q.x, __dp4a(a.y, q.y, __dp4a(a.z, q.z, __dp4a(a.w, q.w, acc[0][t]))));
        acc[1][t] = __dp4a(b.x, q.x, __dp4a(b.y, q.y, __dp4a(b.z, q.z, __dp4a(b.w, q.w, acc[1][t]))));
      }
    }
    int mine = 0;
#pragma unroll
    for (int i = 0; i < 2 * kTokens; ++i) {
      const int sum = __reduce_add_sync(0xFFFFFFFFu, acc[i & 1][i >> 1]);
      if (lane == i) mine = sum;
    }
    const int t = lane >> 1, n = n0 + (lane & 1);
    if (t < tokens && t < kTokens && n < n_out) {
      const float v = (float)mine * token_scale[t] * scales[n];
      if (sizeof(T) == 2) ((__nv_bfloat16*)out)[t * ld_out + n] = __float2bfloat16_rn(v);
      else ((float*)out)[t * ld_out + n] = v;
    }
  }
}

}  // namespace mat
}  // namespace rtopk
