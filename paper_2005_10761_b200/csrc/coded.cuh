// 8-bit codes with one binary32 scale for each row or column, and what makes them.
//
//   s = max |v| / 127,   q = rint(v / s) clamped to +-127      (both quotients rounded to binary32)
//
// over a row (one token, one output channel) or a column (one channel over the tokens).  An all-zero row has s = 0 and
// q = 0; a row with an infinity or a NaN has s = NaN and q = 0, so that everything it takes part in is NaN.
#pragma once

#include "values.cuh"

namespace rtopk {
namespace mat {

__device__ __forceinline__ float code_scale(uint32_t max_magnitude) {
  if (max_magnitude >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  return __fdiv_rn(__uint_as_float(max_magnitude), 127.f);
}
// Codes without a division for each: with r the correctly rounded reciprocal of s and q = v r, the remainder v - q s is exact in a
// fused multiply-add and q + r (v - q s) is the correctly rounded quotient (Markstein, IBM J. Res. Dev. 34, 1990); adding
// 1.5 * 2^23 to it rounds it to a whole number and leaves that in the low byte of the sum.  (Testing how near a plain product
// comes to the middle between two codes does not pay: bfloat16 values over a bfloat16 maximum are quotients of small whole
// numbers, one in three hundred is such a tie.)
struct Coder {
  float s, r;        // the scale and its reciprocal, both times 2^-64 and 2^64 where the scale is small
  float up;          // 1, or 2^64: values are multiplied by it first
  uint32_t mask;     // 0 where the scale is no number: all codes are 0
};
constexpr float kUp = 18446744073709551616.f;
__device__ __forceinline__ Coder coder_of(float s) {
  if (!(s >= 0.f)) return {0.f, 0.f, 1.f, 0u};
  if (s == 0.f) return {0.f, 0.f, 1.f, ~0u};
  const float up = s < 1e-18f ? kUp : 1.f;
  s *= up;
  return {s, __fdiv_rn(1.f, s), up, ~0u};
}
constexpr float kToByte = 12582912.f;
__device__ __forceinline__ uint32_t code_byte(float v, float s, float r) {
  const float q = v * r;
  return __float_as_uint(fmaf(fmaf(-q, s, v), r, q) + kToByte);
}
__device__ __forceinline__ uint32_t pack_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
__device__ __forceinline__ uint32_t code4(float a, float b, float c, float d, const Coder& q) {
  if (q.up != 1.f) {      // a subnormal scale may be so coarse that the largest value is more than 127 of it
    const float top = 127.f * q.s;
    a = fminf(fmaxf(a * q.up, -top), top), b = fminf(fmaxf(b * q.up, -top), top);
    c = fminf(fmaxf(c * q.up, -top), top), d = fminf(fmaxf(d * q.up, -top), top);
  }
  return q.mask & pack_bytes(code_byte(a, q.s, q.r), code_byte(b, q.s, q.r), code_byte(c, q.s, q.r), code_byte(d, q.s, q.r));
}

__device__ __forceinline__ uint2 code8(const float (&v)[8], const Coder& q) {
  return make_uint2(code4(v[0], v[1], v[2], v[3], q), code4(v[4], v[5], v[6], v[7], q));
}
__device__ __forceinline__ void store8(uint2 w, int left, int8_t* out) {
  if (left >= 8) {
    *(uint2*)out = w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) out[i] = (int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
  }
}

// Codes along the rows; kWarps warps per row.  A row is read once and kept in registers as it is in memory (128 bytes a thread);
// what is beyond that is read again for its codes.  With kMul column c is multiplied by mul[c] first.  `padded`: that many codes of a
// row are written, those past its end zero.  `clear`: words that a later launch wants zeroed.  Bound by memory and by the warps
// that fit: 8192 rows of 4096 bfloat16 values 20 us (101 MB, 4.9 TB/s), with factors 31 us.
template <class T, int kWarps, bool kMul>
__global__ void __launch_bounds__(256)
k_code_rows(const T* src, int64_t ld, int rows, int cols, int vec, const float* mul, int mul_vec, int8_t* codes, int64_t ld_codes, int padded, float* scales,
            uint32_t* clear, int64_t clear_words) {
  constexpr int kKeep = 16 / sizeof(T), kSpan = kWarps * 32 * 8;
  __shared__ uint32_t part[8];
  const int group = threadIdx.x / (32 * kWarps), t = threadIdx.x % (32 * kWarps);
  const int row = blockIdx.x * (8 / kWarps) + group;
  const bool in = row < rows;
  launch_wait();
  launch_next();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < clear_words; i += (int64_t)gridDim.x * 256) clear[i] = 0u;      // blocks x 256 may pass 32 bits
  const T* p = src + (int64_t)(in ? row : 0) * ld;
  auto values = [&](const Eight<T>& e, int c, float (&v)[8]) {
    e.widen_to(v);
    if constexpr (kMul) {
      float f[8];
      load8(mul + c, cols - c, mul_vec, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= f[j];
    }
  };
  Eight<T> kept[kKeep];
#pragma unroll
  for (int i = 0; i < kKeep; ++i) {
    const int c = i * kSpan + t * 8;
    if (c < cols) kept[i].load(p + c, cols - c, vec);
  }
  uint32_t m = 0;
  float v[8];
  auto widest = [&](const Eight<T>& e, int c) {
    if constexpr (kMul) {
      values(e, c, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max(m, magnitude(v[j]));
    } else {
      m = e.largest(m);
    }
  };
#pragma unroll
  for (int i = 0; i < kKeep; ++i) {
    const int c = i * kSpan + t * 8;
    if (c >= cols) break;
    widest(kept[i], c);
  }
  for (int c = kKeep * kSpan + t * 8; c < cols; c += kSpan) {
    Eight<T> e;
    e.load(p + c, cols - c, vec);
    widest(e, c);
  }
  if constexpr (!kMul) m = Eight<T>::as_magnitude(m);
  m = __reduce_max_sync(0xFFFFFFFFu, m);
  if constexpr (kWarps > 1) {
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
    __syncthreads();
    m = part[group * kWarps + (threadIdx.x & (kWarps - 1))];
    m = __reduce_max_sync(0xFFFFFFFFu, m);
  }
  if (!in) return;
  const float s = code_scale(m);
  if (t == 0) scales[row] = s;
  const Coder q = coder_of(s);
  int8_t* out = codes + row * ld_codes;
#pragma unroll
  for (int i = 0; i < kKeep; ++i) {
    const int c = i * kSpan + t * 8;
    if (c >= cols) break;
    values(kept[i], c, v);
    store8(code8(v, q), padded - c, out + c);
  }
  for (int c = kKeep * kSpan + t * 8; c < cols; c += kSpan) {
    Eight<T> e;
    e.load(p + c, cols - c, vec);
    values(e, c, v);
    store8(code8(v, q), padded - c, out + c);
  }
  for (int c = (cols + 7) / 8 * 8 + t * 8; c < padded; c += kSpan) store8(make_uint2(0u, 0u), padded - c, out + c);
}

// Up to two matrices of the same number of rows in one launch: the first `tiles` blocks along x take the first.
template <class T>
struct Columns {
  const T* src;
  int64_t ld;
  int cols, vec, tiles;
  uint32_t* max_bits;
  int8_t* codes;       // [cols][ld_codes]
  float* scales;
};

// Largest magnitude of every column (max_bits zeroed before): 256 columns per block, eight threads deep.  Two matrices of 8192 x
// 4096 bfloat16 values 29 us (134 MB, 4.6 TB/s).
template <class T>
__global__ void __launch_bounds__(256) k_col_max(const __grid_constant__ Columns<T> first, const __grid_constant__ Columns<T> second, int rows, int rows_per_block) {
  __shared__ uint32_t part[8][256];
  const bool in_first = (int)blockIdx.x < first.tiles;
  const Columns<T>& q = in_first ? first : second;
  const int tile = in_first ? blockIdx.x : blockIdx.x - first.tiles;
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
  const int c = tile * 256 + x * 8, cols = q.cols;
  const int r0 = blockIdx.y * rows_per_block, r1 = min(rows, r0 + rows_per_block);
  launch_wait();
  launch_next();
  uint32_t m[8] = {};
  if (c < cols) {
    const T* src = q.src;
    const int64_t ld = q.ld;
    const bool vec = q.vec;
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
  const int col = tile * 256 + x * 8 + y;     // entry y * 32 + x
  if (col < cols && best) atomicMax(q.max_bits + col, best);
}

// Codes for each column, written transposed: codes[c][r], scales[c].  128 rows x 64 columns per block; four codes of a
// column are one word, so that a row of the result leaves in 128-byte pieces.  The same two matrices 45 us (201 MB, 4.5 TB/s).
template <class T>
__global__ void __launch_bounds__(256) k_code_cols(const __grid_constant__ Columns<T> first, const __grid_constant__ Columns<T> second, int rows, int64_t ld_codes) {
  __shared__ uint32_t tile[64][33];
  __shared__ Coder coder[64];
  const bool in_first = (int)blockIdx.x < first.tiles;
  const Columns<T>& job = in_first ? first : second;
  const T* src = job.src;
  const int64_t ld = job.ld;
  const int cols = job.cols, vec = job.vec;
  const uint32_t* max_bits = job.max_bits;
  int8_t* codes = job.codes;
  float* scales = job.scales;
  const int c0 = (in_first ? blockIdx.x : blockIdx.x - first.tiles) * 64, r0 = blockIdx.y * 128;
  const int cg = (threadIdx.x & 7) * 8, rg = threadIdx.x >> 3;
  launch_wait();
  launch_next();
  const int left = cols - c0 - cg;
  Eight<T> e[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = r0 + rg * 4 + i;
    e[i].load(src + (int64_t)min(r, rows - 1) * ld + c0 + cg, r < rows ? left : 0, vec);
  }
  if (threadIdx.x < 64) {
    const bool in = c0 + threadIdx.x < cols;
    const float s = in ? code_scale(max_bits[c0 + threadIdx.x]) : 0.f;
    if (in && blockIdx.y == 0) scales[c0 + threadIdx.x] = s;
    coder[(threadIdx.x & 7) * 8 + (threadIdx.x >> 3)] = coder_of(s);      // the eight threads of a row read neighbours
  }
  __syncthreads();
  float v[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) e[i].widen_to(v[i]);
#pragma unroll
  for (int j = 0; j < 8; ++j) tile[cg + j][rg] = code4(v[0][j], v[1][j], v[2][j], v[3][j], coder[j * 8 + (threadIdx.x & 7)]);
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

// codes_t[c][r] = codes[r][c]: 128 rows x 64 columns per block, four codes of a column in a word.
__global__ void __launch_bounds__(256) k_codes_transpose(const int8_t* codes, int64_t ld, int rows, int cols, int8_t* out, int64_t ld_out) {
  __shared__ uint32_t tile[64][33];
  const int c0 = blockIdx.x * 64, r0 = blockIdx.y * 128;
  const int cg = (threadIdx.x & 7) * 8, rg = threadIdx.x >> 3;
  launch_wait();
  launch_next();
  uint2 v[4];      // eight columns of four rows; the row stride is a multiple of 16, so whole vectors exist
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = r0 + rg * 4 + i;
    v[i] = r < rows && c0 + cg < cols ? *(const uint2*)(codes + (int64_t)r * ld + c0 + cg) : make_uint2(0u, 0u);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    auto byte = [&](const uint2& w) { return (j < 4 ? w.x : w.y) >> (8 * (j & 3)); };
    tile[cg + j][rg] = pack_bytes(byte(v[0]), byte(v[1]), byte(v[2]), byte(v[3]));
  }
  __syncthreads();
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
  const int n = min(4, rows - r0 - x * 4);
  for (int c = y; c < 64; c += 8) {
    if (c0 + c >= cols || n <= 0) continue;
    int8_t* p = out + (int64_t)(c0 + c) * ld_out + r0 + x * 4;
    const uint32_t w = tile[c][x];
    if (n == 4) *(uint32_t*)p = w;
    else
      for (int i = 0; i < n; ++i) p[i] = (int8_t)(w >> (8 * i));
  }
}

// A linear layer for a few tokens: reading the codes of W once is all the work, so one launch does everything.  Each block
// codes the tokens for itself (they are small, and come from L2), then each warp takes two output channels at a time: 16 codes
// of W a thread, four-way integer dot products with the tokens' codes in shared memory.  One token through 1500 -> 6000: 6.2 us, which is the
// call itself; through 8192 -> 8192 16.9 us (4.0 TB/s; the tokens' coding comes before the first codes of W).
constexpr int kFewThreads = 256;
constexpr int kFewBytes = 47 * 1024;       // codes of all tokens in shared memory, at most (48 KB with the rest)
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
  Coder q[kTokens];
#pragma unroll
  for (int t = 0; t < kTokens; ++t) {
    uint32_t best = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) best = max(best, part[i][t]);
    const float s = code_scale(best);
    if (threadIdx.x == 0) token_scale[t] = s;
    q[t] = coder_of(s);
  }
  for (int c = threadIdx.x * 8; c < row; c += kFewThreads * 8)
#pragma unroll
    for (int t = 0; t < kTokens; ++t) {
      float v[8];
      load8(x + min(t, tokens - 1) * ld_x + min(c, n_in - 1), max(n_in - c, 0), vec, v);
      *(uint2*)(few_smem + t * row + c) = code8(v, q[t]);
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

// The same for up to eight tokens, whose codes come from a launch before (rows of whole 64s, zero past n_in): 32 output channels a
// block, the contraction dealt out to its eight warps in pieces of 64 codes, integer matrix instructions (16 channels x 8
// tokens x 32 codes) straight from registers.  Reading W is what takes the time here, so nothing of it goes through shared
// memory: a thread's 16 consecutive codes of a channel are two instructions' operands, in an order of the contraction index that
// the tokens' codes follow.  The warps' sums meet in shared memory.  Eight tokens through 8192 -> 8192:
// 17.5 us with the coding launch (3.8 TB/s of codes), through 4096 -> 4096 7.4 us (dot products: 16.0).
constexpr int kTokThreads = 256, kTokChannels = 32;

__device__ __forceinline__ void mma_codes(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <class T>
__global__ void __launch_bounds__(kTokThreads, 2)
k_product_tokens(const int8_t* x, int64_t ld_x, const float* token_scales, const int8_t* codes, int64_t ld_codes, const float* scales, int tokens, int n_out, int n_in, T* out,
                 int64_t ld_out) {
  __shared__ int sums[8][8][kTokChannels + 1];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int n0 = blockIdx.x * kTokChannels;
  const int8_t* w[4];      // channels g, g + 8, g + 16, g + 24; those past the last one read it again
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = codes + min(n0 + g + 8 * i, n_out - 1) * ld_codes;
  const int8_t* p = x + min(g, tokens - 1) * ld_x;
  auto read_w = [&](int k, uint4 (&a)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = k < n_in ? __ldg((const uint4*)(w[i] + k)) : make_uint4(0u, 0u, 0u, 0u);
  };
  constexpr int kAhead = 3, kStep = 8 * 64;
  uint4 a[kAhead][4];
  int k = warp * 64 + q * 16;
#pragma unroll
  for (int j = 0; j < kAhead; ++j) read_w(k + j * kStep, a[j]);      // W is not written by the launch before
  launch_wait();
  launch_next();
  int acc[2][4] = {};
  for (int j0 = 0; j0 * kStep + warp * 64 < n_in; j0 += kAhead)
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int kk = k + (j0 + j) * kStep;
      if ((j0 + j) * kStep + warp * 64 >= n_in) break;
      const uint4 b = *(const uint4*)(p + kk);
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        mma_codes(acc[m], a[j][2 * m].x, a[j][2 * m + 1].x, a[j][2 * m].y, a[j][2 * m + 1].y, b.x, b.y);
        mma_codes(acc[m], a[j][2 * m].z, a[j][2 * m + 1].z, a[j][2 * m].w, a[j][2 * m + 1].w, b.z, b.w);
      }
      read_w(kk + kAhead * kStep, a[j]);
    }
  // acc[m]: channels 16 m + g and + 8, tokens 2 q and + 1
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[warp][2 * q + (e & 1)][16 * m + g + 8 * (e >> 1)] = acc[m][e];
  __syncthreads();
  for (int i = threadIdx.x; i < tokens * kTokChannels; i += kTokThreads) {
    const int t = i / kTokChannels, c = i % kTokChannels, n = n0 + c;
    if (n >= n_out) continue;
    int sum = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += sums[j][t][c];
    const float v = (float)sum * token_scales[t] * scales[n];
    if (sizeof(T) == 2) ((__nv_bfloat16*)out)[t * ld_out + n] = __float2bfloat16_rn(v);
    else ((float*)out)[t * ld_out + n] = v;
  }
}

}  // namespace mat
}  // namespace rtopk
