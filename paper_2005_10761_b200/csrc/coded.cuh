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
// rint(v / s) for finite v and s.  The product with the reciprocal r is within 2^-23 of the quotient, 2e-5 at 127: unless
// it lies that near to the middle between two codes, it rounds to the same one; otherwise the quotient is formed.
__device__ __forceinline__ int code(float v, float s, float r) {
  const float t = v * r;
  float q = rintf(t);
  if (!(fabsf(fabsf(t - q) - 0.5f) > 1e-4f)) q = rintf(__fdiv_rn(v, s));
  return max(-127, min(127, (int)q));
}
// The reciprocal for code(): NaN where the quotient has to be formed every time, 0 (with s = 1) where all codes are 0.
__device__ __forceinline__ float code_reciprocal(float& s) {
  if (!(s > 0.f)) { s = 1.f; return 0.f; }
  return s < 1e-36f ? __uint_as_float(0x7FC00000u) : __fdiv_rn(1.f, s);
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
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i >> 2] |= (uint32_t)(uint8_t)code(v[i], s, r) << (8 * (i & 3));
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
#pragma unroll 4
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
  const int c0 = blockIdx.x * 64, r0 = blockIdx.y * 128;
  const int cg = (threadIdx.x & 7) * 8, rg = threadIdx.x >> 3;
  launch_wait();
  launch_next();
  const int left = cols - c0 - cg;
  float v[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = r0 + rg * 4 + i;
    if (left > 0 && r < rows) load8(src + (int64_t)r * ld + c0 + cg, left, vec, v[i]);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (j >= left) break;
    float s = code_scale(max_bits[c0 + cg + j]);
    if (blockIdx.y == 0 && rg == 0) scales[c0 + cg + j] = s;
    const float r = code_reciprocal(s);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= (uint32_t)(uint8_t)code(v[i][j], s, r) << (8 * i);
    tile[cg + j][rg] = w;
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

}  // namespace mat
}  // namespace rtopk
