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

// Eight neighbours of a row without alignment, of which `left` exist (the others count as zero): the aligned vectors that hold any of them
// are read whole and shifted, and those of several rows are under way before the first is used (4644 x 4086 bfloat16 values 28 -> 22 us).
// Loads of single values, which touch a sector for each lane, took 29.
__device__ __forceinline__ uint4 vector_if(const uint4* p, bool there) { return there ? *p : make_uint4(0u, 0u, 0u, 0u); }
template <class T>
struct Shifted {
  static constexpr int kVectors = sizeof(T) == 4 ? 3 : 2;
  uint4 v[kVectors];
  uint32_t m;      // bytes of the first vector before the first value
  __device__ __forceinline__ void load(const T* p, int left) {
    m = (uint32_t)(uintptr_t)p & 15u;
    const uint4* at = (const uint4*)((uintptr_t)p & ~(uintptr_t)15);
    const int bytes = left > 0 ? (int)m + min(left, 8) * (int)sizeof(T) : 0;      // up to the last one, from the first vector's start
#pragma unroll
    for (int k = 0; k < kVectors; ++k) v[k] = vector_if(at + k, bytes > 16 * k);
  }
  __device__ __forceinline__ void shift(int left, Eight<T>& e) const {
    uint32_t w[4 * kVectors];
    memcpy(w, v, sizeof w);
    constexpr int kWords = 2 * (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < kWords + 2; ++i) w[i] = m & 8u ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < kWords + 1; ++i) w[i] = m & 4u ? w[i + 1] : w[i];
    if constexpr (sizeof(T) == 2) {
      const uint32_t half = m & 2u ? 0x5432u : 0x3210u;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = __byte_perm(w[i], w[i + 1], half);
    }
    if (left < 8)
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        if (sizeof(T) == 4) w[i] = i < left ? w[i] : 0u;
        else if (2 * i + 1 >= left) w[i] &= 2 * i < left ? 0xFFFFu : 0u;
      }
    memcpy(&e, w, sizeof e);
  }
};

// Codes of a tile of 128 x 128 values along its rows (blocks of 32 columns) and, transposed, along its columns (blocks of 32
// rows), the values read once.  kTile: one scale for each 32 x 32 values, the same codes both ways.  A warp takes 32 rows and 64 columns, a
// thread eight neighbours in each of eight rows: the maxima along rows meet in four lanes, those along columns in the other four, and the
// codes of both directions are whole words.  Past the matrix's end codes and scales are zero; a row's codes are written up to a
// whole number of blocks.
// Up to two matrices in one launch: the first `tiles` blocks take the first.
//
// Bound by memory along rows (4096 x 4096 bfloat16 11 us from DRAM under a profiler), both ways by the instructions for bfloat16, issued in 70 % of
// the cycles (two such matrices, one of them both ways, 20 us).  Binary32 weights both ways have neither full: 4096 x 4096 in 32 x 32 tiles 19.0 us,
// 13 at memory's rate, instructions issued in 36 % of the cycles, with a quarter of the warps that an SM holds (98 registers).
template <class T>
struct CodeJob {
  const T* src;
  int64_t ld;
  int rows, cols, vec, tiles_c;
  MicroOut by_row, by_col;      // without codes: not asked for (where the kernel has both)
};

// kAligned: both matrices' rows start on multiples of 16 bytes.
template <class T, bool kRows, bool kColumns, bool kTile, bool kAligned>
__global__ void __launch_bounds__(256)
k_micro_code(const __grid_constant__ CodeJob<T> first, const __grid_constant__ CodeJob<T> second, int tiles) {
  __shared__ uint32_t col_codes[kColumns ? 128 : 1][17];
  __shared__ __align__(16) uint8_t row_scales[512], col_scales[512];
  constexpr int kTogether = sizeof(T) == 4 ? 4 : 8;
  const bool in_first = (int)blockIdx.x < tiles;
  const CodeJob<T>& job = in_first ? first : second;
  const T* src = job.src;
  const int64_t ld = job.ld;
  const int rows = job.rows, cols = job.cols, vec = job.vec, tiles_c = job.tiles_c;
  const MicroOut by_row = job.by_row, by_col = job.by_col;
  const bool along_rows = kRows && (!kColumns || by_row.codes);
  const int tile = in_first ? blockIdx.x : blockIdx.x - tiles;
  const int tile_r = tile / tiles_c, tile_c = tile - tile_r * tiles_c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, cl = lane & 7, rl = lane >> 3;
  const int wr = (warp & 3) * 32, wc = (warp >> 2) * 64;       // the warp's place in the tile
  const int r0 = tile_r * 128 + wr + rl * 8, c0 = tile_c * 128 + wc + cl * 8;
  const bool whole = tile_r * 128 + 128 <= rows && tile_c * 128 + 128 <= cols;
  launch_wait();
  launch_next();
  Eight<T> e[8];
  if (kAligned && whole) {
    const T* p = src + (int64_t)r0 * ld + c0;
#pragma unroll
    for (int i = 0; i < 8; ++i, p += ld) e[i].load(p, 8, true);
  } else if (kAligned || vec) {
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i].load(src + (int64_t)min(r0 + i, rows - 1) * ld + min(c0, cols - 1), r0 + i < rows ? cols - c0 : 0, true);
  } else {
    const T* p = src + (int64_t)r0 * ld + c0;
#pragma unroll
    for (int h = 0; h < 8; h += kTogether) {      // rows whose loads are all under way before the first is used
      Shifted<T> v[kTogether];
#pragma unroll
      for (int i = 0; i < kTogether; ++i, p += ld) v[i].load(p, r0 + h + i < rows ? cols - c0 : 0);
      asm volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < kTogether; ++i) v[i].shift(r0 + h + i < rows ? cols - c0 : 0, e[h + i]);
    }
  }
  uint32_t shared = 0u;
  if constexpr (kTile) {
    shared = micro_scale(Magnitudes<T>::all(e));
  }
  if (along_rows) {
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
  if (along_rows && threadIdx.x < 32) {
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

// ----------------------------------------------------------------------------- a few tokens
// The layer for up to four tokens, where reading W is the work, in one launch.  Every block codes the tokens for itself; then each warp takes four
// channels at a time, 32 apart, whose scales lie together, and a lane a block of 32 codes of each: integer dot products with the tokens'
// codes in shared memory, times the two scales, added in binary32.
//
// A code is looked up as a byte, twice its value plus 12: one byte permutation takes four codes as selectors into the eight bytes of a table,
// in which a code's sign bit asks for a byte's sign instead, 0 here; so the positive codes come from one table, the negative ones, their
// sign bits turned round, from another, and the two are or'ed.  The 12 is taken off the sum: 12 times the sum of the token's codes.
// 1 token through 1500 -> 6000 takes 5.7 us, most of it the call; through 8192 -> 8192 12.2 (36 MB of codes and scales: 5.5 at memory's rate),
// where the look-ups and products are half of the cycles.
constexpr int kFewTokens = 4, kFewAhead = 2;
constexpr uint32_t kFewPositive0 = 0x0F0E0D0Cu, kFewPositive1 = 0x18141210u, kFewNegative0 = 0x090A0B0Cu, kFewNegative1 = 0x00040608u;
__device__ __forceinline__ uint32_t permute(uint32_t a, uint32_t b, uint32_t selectors) {
  uint32_t r;
  asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(selectors));
  return r;
}
// Two words of four bytes from a word of eight codes.
__device__ __forceinline__ void few_bytes(uint32_t w, uint32_t& low, uint32_t& high) {
  const uint32_t turned = w ^ 0x88888888u;
  low = permute(kFewPositive0, kFewPositive1, w) | permute(kFewNegative0, kFewNegative1, turned);
  high = permute(kFewPositive0, kFewPositive1, w >> 16) | permute(kFewNegative0, kFewNegative1, turned >> 16);
}
// 2^(b - 127); infinity for NaN's 255, which makes NaN of its block's zeros.
__device__ __forceinline__ float power_of(uint32_t b) { return __uint_as_float(b ? b << 23 : 1u << 22); }
constexpr int few_smem(int tokens, int64_t n_in) { return (int)((n_in + 31) / 32) * tokens * (32 + 8); }

template <class T, int kTokens>
__global__ void __launch_bounds__(256)
k_micro_few(const T* x, int64_t ld_x, int vec, const __grid_constant__ MicroOut w, int tokens, int n_out, int n_in, T* out, int64_t ld_out) {
  extern __shared__ __align__(16) char few_smem_raw[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int blocks = (n_in + 31) / 32, pieces = (n_in + 255) / 256 * 2;
  uint4* x_codes = (uint4*)few_smem_raw;                                   // [token][half of a block][block]: twice the codes' values, bytes
  uint2* x_scales = (uint2*)(x_codes + 2 * kTokens * blocks);              // [token][block]: a quarter of the scale, 12 times the codes' sum
  const int units = (n_out + 127) / 128 * 32, step = gridDim.x * 8;
  launch_wait();
  launch_next();
  struct Batch { uint4 codes[kFewAhead][4], scales[kFewAhead]; };
  // of blocks first + lane, + 32, ..: four channels' codes, and four blocks' scales of each
  auto read = [&](int unit, int first, Batch& v) {
    const int group = unit >> 5, r = unit & 31;
#pragma unroll
    for (int k = 0; k < kFewAhead; ++k) {
      const int b = first + 32 * k + lane;
      if (b < blocks) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v.codes[k][i] = __ldg((const uint4*)(w.codes + (int64_t)min(group * 128 + r + 32 * i, n_out - 1) * w.ld + b * 16));
        v.scales[k] = __ldg((const uint4*)(w.scales + ((int64_t)group * pieces + (b >> 2)) * 512 + r * 16));
      }
    }
  };
  Batch now, next;
  int unit = blockIdx.x * 8 + warp;
  if (unit < units) read(unit, 0, now);
  for (int i = threadIdx.x; i < kTokens * blocks; i += 256) {
    const int t = i / blocks, b = i - t * blocks;
    uint32_t bytes[8] = {}, scale = 0u;
    int sum = 0;
    if (t < tokens) {
      Eight<T> e[4];
      uint32_t m = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) e[k].load(x + t * ld_x + min(b * 32 + k * 8, n_in - 1), n_in - b * 32 - k * 8, vec);
#pragma unroll
      for (int k = 0; k < 4; ++k) m = e[k].largest(m);
      scale = micro_scale(Eight<T>::as_magnitude(m));
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float v[8];
        e[k].widen_to(v);
        uint32_t low, high;
        few_bytes(micro_code8(v, scale), low, high);
        bytes[2 * k] = __vsub4(low, 0x0C0C0C0Cu), bytes[2 * k + 1] = __vsub4(high, 0x0C0C0C0Cu);
        sum = __dp4a((int)bytes[2 * k], 0x0C0C0C0C, __dp4a((int)bytes[2 * k + 1], 0x0C0C0C0C, sum));
      }
    }
    x_codes[2 * t * blocks + b] = make_uint4(bytes[0], bytes[1], bytes[2], bytes[3]);
    x_codes[(2 * t + 1) * blocks + b] = make_uint4(bytes[4], bytes[5], bytes[6], bytes[7]);
    x_scales[t * blocks + b] = make_uint2(__float_as_uint(power_of(scale)), (uint32_t)sum);
  }
  __syncthreads();
  for (; unit < units; unit += step) {
    float acc[4][kTokens] = {};
    for (int first = 0; first < blocks; first += 32 * kFewAhead) {
      // what comes next, of this unit or of the warp's next one
      if (first + 32 * kFewAhead < blocks) read(unit, first + 32 * kFewAhead, next);
      else if (unit + step < units) read(unit + step, 0, next);
#pragma unroll
      for (int k = 0; k < kFewAhead; ++k) {
        const int b = first + 32 * k + lane;
        if (b >= blocks) break;
        const uint32_t s[4] = {now.scales[k].x, now.scales[k].y, now.scales[k].z, now.scales[k].w};
        int dot[4][kTokens];
        float w_scale[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w_scale[i] = power_of(s[i] >> 8 * (b & 3) & 255u);
#pragma unroll
          for (int t = 0; t < kTokens; ++t) dot[i][t] = 0;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint4 q[kTokens];
#pragma unroll
          for (int t = 0; t < kTokens; ++t) q[t] = x_codes[(2 * t + h) * blocks + b];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t a[4];
            few_bytes(h ? now.codes[k][i].z : now.codes[k][i].x, a[0], a[1]);
            few_bytes(h ? now.codes[k][i].w : now.codes[k][i].y, a[2], a[3]);
#pragma unroll
            for (int t = 0; t < kTokens; ++t)
              dot[i][t] = __dp4a((int)a[0], (int)q[t].x, __dp4a((int)a[1], (int)q[t].y, __dp4a((int)a[2], (int)q[t].z, __dp4a((int)a[3], (int)q[t].w, dot[i][t]))));
          }
        }
#pragma unroll
        for (int t = 0; t < kTokens; ++t) {
          const uint2 m = x_scales[t * blocks + b];
          const float x_scale = __uint_as_float(m.x);
#pragma unroll
          for (int i = 0; i < 4; ++i)      // the smaller scale first, so that only what is too large in the end overflows
            acc[i][t] = fmaf((float)(dot[i][t] - (int)m.y) * 0.25f * fminf(x_scale, w_scale[i]), fmaxf(x_scale, w_scale[i]), acc[i][t]);
        }
      }
      now = next;
    }
    float result = 0.f;      // of channel lane & 3 and token lane >> 2
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < kTokens; ++t) {
#pragma unroll
        for (int k = 16; k; k >>= 1) acc[i][t] += __shfl_xor_sync(0xFFFFFFFFu, acc[i][t], k);
        if (lane == t * 4 + i) result = acc[i][t];
      }
    const int t = lane >> 2, n = (unit >> 5) * 128 + (unit & 31) + 32 * (lane & 3);
    if (t < kTokens && t < tokens && n < n_out) {
      if (sizeof(T) == 2) ((__nv_bfloat16*)out)[t * ld_out + n] = __float2bfloat16_rn(result);
      else ((float*)out)[t * ld_out + n] = result;
    }
  }
}

}  // namespace mat
}  // namespace rtopk
