// 4-bit codes with a power of two for every 32 along the contraction index, and what makes them.
//
// A block of 32 values (the last of a row may be shorter) has the scale 2^e, e the least whole number for which no magnitude is
// above 6 2^e, -127 at least; its codes are v / 2^e, which is exact, rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
// negatives, ties to the even code (sign, two bits of exponent, one of mantissa).  Two codes are a byte, the first in its low half.  The
// scale is the byte e + 127; a block with an infinity or a NaN has 255, which counts as NaN, and zeros.
//
// Scales lie as the tensor core takes them: 512 bytes for 128 rows and 128 codes of the contraction index, in which row r's four are
// the bytes from 16 (r mod 32) + 4 (r / 32); such pieces of 128 rows follow one another along the contraction index, an even number of them.
#pragma once

#include "values.cuh"

namespace rtopk {
namespace mat {

// From the largest magnitude's bits.  6 = 1.5 2^2: adding just less than half a mantissa carries where the mantissa is above 1.5.
__device__ __forceinline__ uint32_t micro_scale(uint32_t max_magnitude) {
  const int e = max((int)((max_magnitude + 0x3FFFFFu) >> 23) - 2, 0);
  return max_magnitude >= 0x7F800000u ? 255u : (uint32_t)e;
}
// 1 / 2^e; NaN's codes are made zero by its caller.
__device__ __forceinline__ float micro_factor(uint32_t scale) { return __uint_as_float((254u - min(scale, 254u)) << 23); }

// Eight codes, the first lowest.
__device__ __forceinline__ uint32_t micro_pack(const float (&v)[8]) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}
__device__ __forceinline__ uint32_t micro_code8(const float (&v)[8], uint32_t scale) {
  const float f = micro_factor(scale);
  float q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = v[i] * f;
  return scale == 255u ? 0u : micro_pack(q);
}

struct MicroOut {
  uint8_t *codes, *scales;
  int64_t ld;            // bytes from row to row of the codes
};

// The larger magnitude, NaN if there is one.  Three numbers at a time; or two 16-bit ones in a word (whose signs mean nothing).
__device__ __forceinline__ float max_abs(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ uint32_t max_abs2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t other(uint32_t v, int lanes) { return __shfl_xor_sync(0xFFFFFFFFu, v, lanes); }

// Bits of the largest magnitudes of eight rows' and eight columns' values in a thread's 8 x 8, then over the lanes that share the rows (1, 2:
// 32 columns) and the columns (8, 16: 32 rows); `all`: of all of it.
template <class T>
struct Magnitudes;
template <>
struct Magnitudes<float> {
  using E = Eight<float>;
  static __device__ __forceinline__ float row(const E& e, float m) { return max_abs(max_abs(e.a.x, e.a.y, e.a.z), max_abs(e.a.w, e.b.x, e.b.y), max_abs(e.b.z, e.b.w, m)); }
  static __device__ __forceinline__ void rows(const E (&e)[8], uint32_t (&m)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      m[i] = __float_as_uint(row(e[i], 0.f));
      m[i] = max(m[i], other(m[i], 1));
      m[i] = max(m[i], other(m[i], 2));
    }
  }
  static __device__ __forceinline__ void columns(const E (&e)[8], uint32_t (&m)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      m[j] = __float_as_uint(max_abs(max_abs(e[0].at(j), e[1].at(j), e[2].at(j)), max_abs(e[3].at(j), e[4].at(j), e[5].at(j)), max_abs(e[6].at(j), e[7].at(j), 0.f)));
      m[j] = max(m[j], other(m[j], 8));
      m[j] = max(m[j], other(m[j], 16));
    }
  }
  static __device__ __forceinline__ uint32_t all(const E (&e)[8]) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = row(e[i], m);
    uint32_t bits = __float_as_uint(m);
#pragma unroll
    for (int k : {1, 2, 8, 16}) bits = max(bits, other(bits, k));
    return bits;
  }
};
template <>
struct Magnitudes<__nv_bfloat16> {
  using E = Eight<__nv_bfloat16>;
  static __device__ __forceinline__ uint32_t row(const E& e) { return max_abs2(max_abs2(e.w[0], e.w[1]), max_abs2(e.w[2], e.w[3])); }
  static __device__ __forceinline__ void rows(const E (&e)[8], uint32_t (&m)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const uint32_t a = row(e[i]), b = row(e[i + 1]);
      uint32_t q = max_abs2(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));      // row i's low, row i + 1's high
      q = max_abs2(q, other(q, 1));
      q = max_abs2(q, other(q, 2));
      m[i] = q << 16 & 0x7FFFFFFFu, m[i + 1] = q & 0x7FFF0000u;
    }
  }
  static __device__ __forceinline__ void columns(const E (&e)[8], uint32_t (&m)[8]) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const int k = j / 2;
      uint32_t q = max_abs2(max_abs2(max_abs2(e[0].w[k], e[1].w[k]), max_abs2(e[2].w[k], e[3].w[k])), max_abs2(max_abs2(e[4].w[k], e[5].w[k]), max_abs2(e[6].w[k], e[7].w[k])));
      q = max_abs2(q, other(q, 8));
      q = max_abs2(q, other(q, 16));
      m[j] = q << 16 & 0x7FFFFFFFu, m[j + 1] = q & 0x7FFF0000u;
    }
  }
  static __device__ __forceinline__ uint32_t all(const E (&e)[8]) {
    uint32_t q = row(e[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) q = max_abs2(q, row(e[i]));
#pragma unroll
    for (int k : {1, 2, 8, 16}) q = max_abs2(q, other(q, k));
    return max(q << 16 & 0x7FFFFFFFu, q & 0x7FFF0000u);
  }
};
// Hides what is known of the values, so that they are widened where they are used and not kept in that form.
__device__ __forceinline__ void forget(Eight<float>&) {}
__device__ __forceinline__ void forget(Eight<__nv_bfloat16>& e) { asm volatile("" : "+r"(e.w[0]), "+r"(e.w[1]), "+r"(e.w[2]), "+r"(e.w[3])); }

// Codes of a tile of 128 x 128 values along its rows (blocks of 32 columns) and, transposed, along its columns (blocks of 32
// rows), the values read once.  kTile: one scale for each 32 x 32 values, the same codes both ways.  A warp takes 32 rows and 64 columns, a
// thread eight neighbours in each of eight rows: the maxima along rows meet in four lanes, those along columns in the other four, and the
// codes of both directions are whole words.  Past the matrix's end codes and scales are zero; a row's codes are written up to a
// whole number of blocks.
template <class T, bool kRows, bool kColumns, bool kTile>
__global__ void __launch_bounds__(256)
k_micro_code(const T* src, int64_t ld, int rows, int cols, int vec, int tiles_c, const __grid_constant__ MicroOut by_row, const __grid_constant__ MicroOut by_col) {
  __shared__ uint32_t col_codes[kColumns ? 128 : 1][17];
  __shared__ __align__(16) uint8_t row_scales[512], col_scales[512];
  const int tile_r = blockIdx.x / tiles_c, tile_c = blockIdx.x - tile_r * tiles_c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, cl = lane & 7, rl = lane >> 3;
  const int wr = (warp & 3) * 32, wc = (warp >> 2) * 64;       // the warp's place in the tile
  const int r0 = tile_r * 128 + wr + rl * 8, c0 = tile_c * 128 + wc + cl * 8;
  const bool whole = tile_r * 128 + 128 <= rows && tile_c * 128 + 128 <= cols;
  launch_wait();
  launch_next();
  Eight<T> e[8];
  if (whole && vec) {
    const T* p = src + (int64_t)r0 * ld + c0;
#pragma unroll
    for (int i = 0; i < 8; ++i, p += ld) e[i].load(p, 8, true);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i].load(src + (int64_t)min(r0 + i, rows - 1) * ld + min(c0, cols - 1), r0 + i < rows ? cols - c0 : 0, vec);
  }
  uint32_t shared = 0u;
  if constexpr (kTile) {
    shared = micro_scale(Magnitudes<T>::all(e));
  }
  if constexpr (kRows) {
    uint32_t s[8];
    if constexpr (!kTile) Magnitudes<T>::rows(e, s);
    uint8_t* out = by_row.codes + (int64_t)r0 * by_row.ld + c0 / 2;
    // row r0 + i's scale for these 32 columns: the rows of a lane follow one another
    uint8_t* scale = row_scales + rl * 128 + (wr >> 5) * 4 + (wc + cl * 8) / 32;
    const bool first = (cl & 3) == 0, on = (c0 & ~31) < cols;
#pragma unroll
    for (int i = 0; i < 8; ++i, out += by_row.ld) {
      const uint32_t q = kTile ? shared : micro_scale(s[i]);
      float v[8];
      e[i].widen_to(v);
      const uint32_t w = micro_code8(v, q);
      if (first) scale[i * 16] = (uint8_t)q;
      if (whole || (r0 + i < rows && on)) *(uint32_t*)out = w;
    }
  }
  if constexpr (kRows && kColumns)
#pragma unroll
    for (int i = 0; i < 8; ++i) forget(e[i]);
  if constexpr (kColumns) {
    uint32_t s[8];
    if constexpr (!kTile) Magnitudes<T>::columns(e, s);
    const int c = wc + cl * 8;
    uint8_t* scale = col_scales + (c & 31) * 16 + (c >> 5) * 4 + (wr >> 5);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t q = kTile ? shared : micro_scale(s[j]);
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = e[i].at(j);
      col_codes[c + j][(wr >> 3) + rl] = micro_code8(v, q);
      if (rl == 0) scale[j * 16] = (uint8_t)q;
    }
  }
  __syncthreads();
  // Scales in whole pieces of 512 bytes; where the last piece along a row has an even number, an empty one follows.
  const int pieces_c = (cols + 255) / 256 * 2, pieces_r = (rows + 255) / 256 * 2;
  if (kRows && threadIdx.x < 32) {
    uint4* to = (uint4*)(by_row.scales + ((int64_t)tile_r * pieces_c + tile_c) * 512) + threadIdx.x;
    to[0] = ((const uint4*)row_scales)[threadIdx.x];
    if (tile_c + 1 == tiles_c && tiles_c < pieces_c) to[32] = make_uint4(0u, 0u, 0u, 0u);
  }
  if constexpr (kColumns) {
    if (threadIdx.x >= 32 && threadIdx.x < 64) {
      const int t = threadIdx.x - 32, tiles_r = (rows + 127) / 128;
      uint4* to = (uint4*)(by_col.scales + ((int64_t)tile_c * pieces_r + tile_r) * 512) + t;
      to[0] = ((const uint4*)col_scales)[t];
      if (tile_r + 1 == tiles_r && tiles_r < pieces_r) to[32] = make_uint4(0u, 0u, 0u, 0u);
    }
    for (int i = threadIdx.x; i < 512; i += 256) {
      const int c = i >> 2, part = i & 3;      // 16 bytes: a block of 32 rows
      if (whole || (tile_c * 128 + c < cols && tile_r * 128 + part * 32 < rows)) {
        const uint32_t* w = &col_codes[c][part * 4];
        *(uint4*)(by_col.codes + (int64_t)(tile_c * 128 + c) * by_col.ld + tile_r * 64 + part * 16) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
}

}  // namespace mat
}  // namespace rtopk
