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

__device__ __forceinline__ uint32_t micro_scale(uint32_t max_magnitude) {
  if (max_magnitude >= 0x7F800000u) return 255u;
  const int e = (int)(max_magnitude >> 23) - 2 + ((max_magnitude & 0x7FFFFFu) > 0x400000u);      // 6 = 1.5 2^2
  return (uint32_t)max(e, 0);
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
  launch_wait();
  launch_next();
  Eight<T> e[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i].load(src + (int64_t)min(r0 + i, rows - 1) * ld + min(c0, cols - 1), r0 + i < rows ? cols - c0 : 0, vec);
  uint32_t row_scale[8], col_scale[8];
  if constexpr (kTile) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = e[i].largest(m);
    m = Eight<T>::as_magnitude(m);
#pragma unroll
    for (int k : {1, 2, 8, 16}) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, k));
    const uint32_t s = micro_scale(m);
#pragma unroll
    for (int i = 0; i < 8; ++i) row_scale[i] = col_scale[i] = s;
  } else {
    if constexpr (kRows) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t m = Eight<T>::as_magnitude(e[i].largest(0));
        m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
        m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
        row_scale[i] = micro_scale(m);
      }
    }
    if constexpr (kColumns) {
      uint32_t m[8] = {};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float v[8];
        e[i].widen_to(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) m[j] = max(m[j], magnitude(v[j]));
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        m[j] = max(m[j], __shfl_xor_sync(0xFFFFFFFFu, m[j], 8));
        m[j] = max(m[j], __shfl_xor_sync(0xFFFFFFFFu, m[j], 16));
        col_scale[j] = micro_scale(m[j]);
      }
    }
  }
  if constexpr (kRows) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float v[8];
      e[i].widen_to(v);
      const uint32_t w = micro_code8(v, row_scale[i]);
      const int r = wr + rl * 8 + i;
      if ((cl & 3) == 0) row_scales[(r & 31) * 16 + (r >> 5) * 4 + (wc + cl * 8) / 32] = (uint8_t)row_scale[i];
      if (r0 + i < rows && (c0 & ~31) < cols) *(uint32_t*)(by_row.codes + (r0 + i) * by_row.ld + c0 / 2) = w;
    }
  }
  if constexpr (kColumns) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float u[8];
        e[i].widen_to(u);
        v[i] = u[j];
      }
      const int c = wc + cl * 8 + j;
      col_codes[c][(wr >> 3) + rl] = micro_code8(v, col_scale[j]);
      if (rl == 0) col_scales[(c & 31) * 16 + (c >> 5) * 4 + (wr >> 5)] = (uint8_t)col_scale[j];
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
      if (tile_c * 128 + c < cols && tile_r * 128 + part * 32 < rows) {
        const uint32_t* w = &col_codes[c][part * 4];
        *(uint4*)(by_col.codes + (int64_t)(tile_c * 128 + c) * by_col.ld + tile_r * 64 + part * 16) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
}

}  // namespace mat
}  // namespace rtopk
