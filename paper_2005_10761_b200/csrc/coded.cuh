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
__device__ __forceinline__ int code(float v, float s) {
  if (!(s > 0.f)) return 0;
  const int q = __float2int_rn(__fdiv_rn(v, s));
  return max(-127, min(127, q));
}

// One block per row: codes along the row.  `mul` (may be null) multiplies column c first.
template <class T>
__global__ void __launch_bounds__(256) k_code_rows(const T* src, int64_t ld, int cols, const float* mul, int8_t* codes, int64_t ld_codes, float* scales) {
  __shared__ uint32_t part[8];
  launch_wait();
  launch_next();
  const T* row = src + blockIdx.x * ld;
  uint32_t m = 0;
  for (int c = threadIdx.x; c < cols; c += blockDim.x) m = max(m, magnitude(mul ? widen(row[c]) * mul[c] : widen(row[c])));
  m = __reduce_max_sync(0xFFFFFFFFu, m);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
  __syncthreads();
  m = part[threadIdx.x & 7];
  m = __reduce_max_sync(0xFFFFFFFFu, m);
  const float s = code_scale(m);
  if (threadIdx.x == 0) scales[blockIdx.x] = s;
  int8_t* out = codes + blockIdx.x * ld_codes;
  for (int c = threadIdx.x; c < cols; c += blockDim.x) out[c] = (int8_t)code(mul ? widen(row[c]) * mul[c] : widen(row[c]), s);
}

// Largest magnitude of every column (max_bits zeroed before).
template <class T>
__global__ void __launch_bounds__(256) k_col_max(const T* src, int64_t ld, int rows, int cols, int rows_per_block, uint32_t* max_bits) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  const int r0 = blockIdx.y * rows_per_block, r1 = min(rows, r0 + rows_per_block);
  launch_wait();
  launch_next();
  if (c >= cols) return;
  uint32_t m = 0;
  for (int r = r0; r < r1; ++r) m = max(m, magnitude(widen(src[r * ld + c])));
  if (m) atomicMax(max_bits + c, m);
}

// Codes for each column, written transposed: codes[c][r], scales[c].
template <class T>
__global__ void __launch_bounds__(256) k_code_cols(const T* src, int64_t ld, int rows, int cols, const uint32_t* max_bits, int8_t* codes, int64_t ld_codes, float* scales) {
  __shared__ int8_t tile[64][65];
  const int c0 = blockIdx.x * 64, r0 = blockIdx.y * 64;
  launch_wait();
  launch_next();
  const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
  const float s = c0 + x < cols ? code_scale(max_bits[c0 + x]) : 0.f;
  if (blockIdx.y == 0 && y == 0 && c0 + x < cols) scales[c0 + x] = s;
  for (int r = y; r < 64; r += 4)
    if (r0 + r < rows && c0 + x < cols) tile[x][r] = (int8_t)code(widen(src[(int64_t)(r0 + r) * ld + c0 + x]), s);
  __syncthreads();
  for (int c = y; c < 64; c += 4)
    if (c0 + c < cols && r0 + x < rows) codes[(int64_t)(c0 + c) * ld_codes + r0 + x] = tile[c][x];
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
