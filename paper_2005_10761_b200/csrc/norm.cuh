// Operators along the rows of a worker's activations: dropout from a counter-based generator, and layer normalisation with the
// dropout and the residual sum before it, forwards and backwards.
//
//   t = residual + D(x);   y = gamma (t - mean) rstd + beta                       mean and variance over the row
//   dt = rstd (g - mean(g) - h mean(g h)) + dtotal,  g = gamma dy, h = (t - mean) rstd;   dx = D(dt)
//   dgamma = sum over the rows of dy h,   dbeta = sum over the rows of dy
//
// All of it is bound by memory.  Forwards a row that fits a block is read once and kept in registers between its sums and its results; the gradients
// read it from shared memory for its sums and again for its results; of longer rows what does not fit is read from memory again.
#pragma once

#include "common.cuh"
#include "grids.h"
#include "values.cuh"

namespace rtopk {
namespace mat {

// ----------------------------------------------------------------------------- dropout's mask
// Eight neighbours of a row take the eight 16-bit halves of one Philox4x32-10 output, so that a number costs an eighth of
// ten rounds; p is a multiple of 2^-16 therefore.
struct Mask {
  uint32_t limit;            // an element whose number is below is dropped; 0: there is no mask
  float factor;              // of those that are kept
  uint32_t tag;              // 2^31 + 2^16 site + worker, which no draw of the sampler has
  uint32_t keys[20];         // two for each round
  uint32_t step;
  const uint32_t* step_ptr;  // added to step when the kernel runs
};
__device__ __forceinline__ uint32_t mask_step(const Mask& m) { return m.step + (m.limit && m.step_ptr ? *m.step_ptr : 0u); }
// Columns 8 group .. 8 group + 7: the column at j is kept if its half of the words is not below the limit.
__device__ __forceinline__ uint4 mask_words(const Mask& m, uint32_t step, uint32_t row, uint32_t group) {
  return philox4x32_10(group, row, m.tag, step, m.keys);
}
__device__ __forceinline__ void drop8(const Mask& m, const uint4& x, float (&v)[8]) {
  const uint32_t t = m.limit * 0x10001u, w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    bool low, high;
    __vibmax_u16x2(w[j], t, &high, &low);      // which halves are not below the limit
    v[2 * j] = low ? v[2 * j] * m.factor : 0.f;
    v[2 * j + 1] = high ? v[2 * j + 1] * m.factor : 0.f;
  }
}
// Bit j: column 8 group + j is kept.
__device__ __forceinline__ uint32_t kept8(const Mask& m, uint32_t step, uint32_t row, uint32_t group) {
  const uint4 x = mask_words(m, step, row, group);
  const uint32_t t = m.limit << 16;
  auto two = [&](uint32_t w) { return (w << 16 >= t ? 1u : 0u) | (w >= t ? 2u : 0u); };
  return two(x.x) | two(x.y) << 2 | two(x.z) << 4 | two(x.w) << 6;
}

// ----------------------------------------------------------------------------- eight values of a row in a thread
// A warp takes 256 columns from `base`.  kVec: rows of whole vectors (a multiple of eight columns), of which a thread has eight neighbours or
// none; else a thread has every 32nd column, so that loads and stores of rows without alignment are coalesced.
constexpr int kWarpCols = 256;
template <bool kVec>
__device__ __forceinline__ int col_of(int base, int lane, int j) { return kVec ? base + lane * 8 + j : base + j * 32 + lane; }
// Whether the thread has any of the columns; without kVec the warp does.
template <bool kVec>
__device__ __forceinline__ bool has_cols(int base, int lane, int cols) { return kVec ? base + lane * 8 < cols : base < cols; }

// 32 bytes at once, so that a sector is asked for and written in one piece.
__device__ __forceinline__ void load_vector(const float* p, Eight<float>& e) {
  asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(e.a.x), "=f"(e.a.y), "=f"(e.a.z), "=f"(e.a.w), "=f"(e.b.x), "=f"(e.b.y), "=f"(e.b.z), "=f"(e.b.w)
               : "l"(p)
               : "memory");
}
__device__ __forceinline__ void load_vector(const __nv_bfloat16* p, Eight<__nv_bfloat16>& e) { e.load(p, 8, true); }

template <class T, bool kVec>
__device__ __forceinline__ void load_cols(const T* row, int base, int lane, int cols, Eight<T>& e) {
  if constexpr (kVec) {
    if (has_cols<true>(base, lane, cols)) load_vector(row + base + lane * 8, e);
  } else if constexpr (sizeof(T) == 4) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = base + j * 32 + lane < cols ? (float)row[base + j * 32 + lane] : 0.f;
    e.a = make_float4(v[0], v[1], v[2], v[3]), e.b = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    const uint16_t* u = (const uint16_t*)row;
    uint32_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = base + j * 32 + lane < cols ? u[base + j * 32 + lane] : 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) e.w[j] = v[2 * j] | v[2 * j + 1] << 16;
  }
}
template <bool kVec>
__device__ __forceinline__ void load_cols(const float* row, int base, int lane, int cols, float (&v)[8]) {
  Eight<float> e = {};
  load_cols<float, kVec>(row, base, lane, cols, e);
  e.widen_to(v);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
               : "memory");
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
  __nv_bfloat162 q[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) q[j] = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
  uint4 w;
  memcpy(&w, q, sizeof w);
  *(uint4*)p = w;
}
__device__ __forceinline__ void narrow(float v, float& out) { out = v; }
__device__ __forceinline__ void narrow(float v, __nv_bfloat16& out) { out = __float2bfloat16_rn(v); }
// kVec: for threads that have columns.
template <class T, bool kVec>
__device__ __forceinline__ void store_cols(T* row, int base, int lane, int cols, const float (&v)[8]) {
  if constexpr (kVec) {
    store8(row + base + lane * 8, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (base + j * 32 + lane < cols) narrow(v[j], row[base + j * 32 + lane]);
  }
}
// v <- D(v) for the warp's 256 columns from `base`.
template <bool kVec>
__device__ __forceinline__ void drop_cols(const Mask& m, uint32_t step, uint32_t row, int base, int lane, float (&v)[8]) {
  const uint32_t group = (uint32_t)base / 8 + lane;
  if constexpr (kVec) {
    drop8(m, mask_words(m, step, row, group), v);
  } else {
    const uint32_t own = kept8(m, step, row, group);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __shfl_sync(0xFFFFFFFFu, own, 4 * j + (lane >> 3)) >> (lane & 7) & 1 ? v[j] * m.factor : 0.f;
  }
}

__device__ __forceinline__ float sum8(const float (&v)[8]) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int k = 16; k; k >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, k);
  return v;
}
// 1 / sqrt(v), the approximation improved by one Newton step: within 2 steps of binary32.  0 of infinity and infinity of 0: there the step's
// residual is NaN, of which fminf makes a number that changes neither.
__device__ __forceinline__ float inverse_root(float v) {
  const float r = rsqrtf(v);
  return fmaf(r * fminf(fmaf(-v * r, r, 1.f), 1.f), 0.5f, r);
}
// The sum over the block; `part` has a place for each warp and is used once between two barriers.
__device__ __forceinline__ float row_sum(float v, float* part) {
  const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  v = warp_sum(v);
  if (lane == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  return warp_sum(lane < warps ? part[lane] : 0.f);
}

// ----------------------------------------------------------------------------- dropout
__device__ __forceinline__ uint32_t divide(uint32_t k, const Divisor& v) { return v.d == 1 ? k : __umulhi(k, v.m) >> v.shift; }

// Four rows at a time: a thread takes eight neighbouring columns of them (kVec), or a warp 256, so that what the generator's first
// rounds make of the column is shared by four rows.  Bands of `band` rows, a multiple of four, along the grid's second side.
//
// A share of memory's rate is left to the generator's multiplications, which run at a quarter of the usual rate: 8192 x 16384 bfloat16 94.8 us,
// 5.7 TB/s (a copy: 6.5); one row a thread took 112.
template <class T, bool kVec>
__global__ void __launch_bounds__(256) k_dropout(const T* x, int64_t ld_x, int64_t rows, int cols, int64_t band, const Divisor units, const __grid_constant__ Mask mask, T* out, int64_t ld_out) {
  constexpr int kEach = 4;
  const uint32_t k = kVec ? blockIdx.x * 256u + threadIdx.x : blockIdx.x * 8u + (threadIdx.x >> 5);
  const uint32_t quad = divide(k, units), unit = k - quad * units.d;
  const int64_t row = blockIdx.y * band + (int64_t)quad * kEach;
  const int left = (int)min((int64_t)kEach, min(rows, (blockIdx.y + 1) * band) - row);
  const int base = kVec ? (int)unit * 8 : (int)unit * kWarpCols, lane = kVec ? 0 : threadIdx.x & 31;
  launch_wait();
  launch_next();
  if (left <= 0) return;
  const uint32_t step = mask_step(mask);
  const T* from = x + row * ld_x;
  T* to = out + row * ld_out;
  Eight<T> e[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i)
    if (i < left) load_cols<T, kVec>(from + i * ld_x, base, lane, cols, e[i]);
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    if (i >= left) break;
    float v[8];
    e[i].widen_to(v);
    drop_cols<kVec>(mask, step, (uint32_t)(row + i), base, lane, v);
    store_cols<T, kVec>(to + i * ld_out, base, lane, cols, v);
  }
}

// ----------------------------------------------------------------------------- layer normalisation
template <class T>
struct NormArgs {
  const T *x, *residual;      // residual, total, mean, rstd, gamma, beta may be null
  T *y, *total;
  int64_t ld_x, ld_r, ld_y, ld_t;
  const float *gamma, *beta;
  float *mean, *rstd;
  int rows, cols;
  float eps;
  Mask mask;
};

// Rows that fit the block are taken in turn: one block per SM, `rows_per` rows of it at a time with `warps` warps each (a group), kKeep pieces of
// 256 columns a warp.  What a thread needs of the next rows is on its way to its own place in shared memory (kVec: asynchronous copies,
// kStages rows deep; else by way of registers).  A row's sums meet while the results of the row before are formed, so that neither the
// barrier nor the sums' latency stops the block; one barrier a row, of the row's warps.
//
// The bound is memory as long as the instructions keep up: 16 columns a thread, so that a row's sums, addresses and statistics are shared
// by 16, and places in shared memory that differ by constants.  Bfloat16 with dropout and residual sum: 8192 x 4096 51.8 us; gradients of
// 16384 x 8192 258 us (5.2 TB/s both; instructions are issued in 61 and 64 % of the cycles).  A block for each row took 417 for the latter.
// Widths that do not fill the block's 16 warps leave some of that: 8192 x 4608, 9 warps, 79 us, and rows of one piece most of it: 262144 x 64
// without dropout and residual 106 us.  Without alignment values are loaded one by one: 8192 x 4095 121 us.  Binary32 rows of 8193 to 16384 columns
// with a residual have one stage, so that nothing is on its way during a row's sums: 4096 x 16384 294 us, 3.7 TB/s.
constexpr int kRowWarps = 16, kRowSmem = 216 * 1024;
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// For the warp's copies but the last kLeft groups of each thread.
template <int kLeft>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
  __syncwarp();
}

template <class T, bool kVec, int kKeep, int kArrays>
struct RowShape {
  static constexpr int kPlanes = sizeof(T) / 2;                       // a thread's eight values lie in pieces of 16 bytes,
  static constexpr int kPlane = 32 * kRowWarps * 16;                  // each thread's next to the others'
  static constexpr int kStage = kArrays * kKeep * kPlanes * kPlane;
  static constexpr int kFit = kRowSmem / kStage, kStages = kVec ? (kFit > 4 ? 4 : kFit) : 1;
  static constexpr int kSmem = kStages * kStage;
};

// kFull (with kVec): the row is just what its warps hold, so that every thread has all of its columns.  With kVec a row's work is one run of code
// without branches: threads without columns go along with zeros.
template <class T, bool kVec, bool kFull, int kKeep, int kArrays>
struct RowPipe : RowShape<T, kVec, kKeep, kArrays> {
  using S = RowShape<T, kVec, kKeep, kArrays>;
  using S::kPlanes;
  using S::kPlane;
  using S::kStage;
  using S::kStages;
  int warps, group, in_row, lane, cols;
  int count, first, step;      // rows of the group, the first of them, and how far apart they are
  int fetched, to;             // rows on their way or here, and the stage of the next
  char* mine;
  struct Source {
    const T* p;                // of the next row to be read
    int64_t step;
    Eight<T> next[kVec ? 1 : kKeep];
  } s0, s1, s2;

  __device__ __forceinline__ RowPipe(char* smem, int warps, int rows_per, int rows, int cols) : warps(warps), cols(cols) {
    lane = threadIdx.x & 31;
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0);
    group = warp / warps, in_row = warp - group * warps;
    first = blockIdx.x * rows_per + group, step = gridDim.x * rows_per;
    count = first < rows ? (rows - 1 - first) / step + 1 : 0;
    mine = smem + threadIdx.x * 16;
    fetched = to = 0;
  }
  __device__ __forceinline__ int base(int i) const { return (i * warps + in_row) * kWarpCols; }
  // Whether piece i is to be worked on: without kVec where the warp has columns of it.
  __device__ __forceinline__ bool works(int i) const { return kVec || on(i); }
  __device__ __forceinline__ bool on(int i) const { return kFull || has_cols<kVec>(base(i), lane, cols); }
  __device__ __forceinline__ char* place(int stage, int q, int i) const { return mine + stage * kStage + (q * kKeep + i) * kPlanes * kPlane; }
  __device__ __forceinline__ void source(Source& s, const T* p, int64_t ld) { s.p = p + first * ld + (kVec ? base(0) : 0), s.step = ld * step; }
  __device__ __forceinline__ void fetch(Source& s, int q) {
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
      if constexpr (kVec) {
        // Neighbouring lanes copy neighbouring pieces of 16 bytes; of binary32 values that is not the thread's own, but its warp's.
#pragma unroll
        for (int r = 0; r < kPlanes; ++r) {
          const int piece = r * 32 + lane, owner = piece / kPlanes;
          if (kFull || base(i) + owner * 8 < cols)
            copy16(smem_addr(place(to, q, i)) + (owner - lane) * 16 + (piece % kPlanes) * kPlane, (const char*)(s.p + i * warps * kWarpCols) + 16 * piece);
        }
      } else {
        load_cols<T, false>(s.p, base(i), lane, cols, s.next[i]);
      }
    }
    s.p += s.step;
  }
  __device__ __forceinline__ void fetch() {
    if constexpr (kVec && kPlanes > 1) __syncwarp();      // the place has been read by all of the warp
    if (fetched < count) {
      fetch(s0, 0);
      if (kArrays > 1) fetch(s1, 1);
      if (kArrays > 2) fetch(s2, 2);
    }
    ++fetched;
    if constexpr (kVec) {
      copies_commit();
      to = to + 1 == kStages ? 0 : to + 1;
    }
  }
  __device__ __forceinline__ void start(int rows) {
    if constexpr (kVec && !kFull) {      // places that no copy fills: threads without columns go along with zeros
#pragma unroll
      for (int i = 0; i < kKeep; ++i)
        if (!on(i))
          for (int s = 0; s < kStages; ++s)
#pragma unroll
            for (int q = 0; q < kArrays * kPlanes; ++q) *(uint4*)(place(s, q / kPlanes, i) + q % kPlanes * kPlane) = make_uint4(0u, 0u, 0u, 0u);
      __syncwarp();
    }
    for (int k = 0; k < rows; ++k) fetch();
  }
  __device__ __forceinline__ void land(const Source& s, int q) {
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
      uint4 w[kPlanes];
      memcpy(w, &s.next[i], sizeof w);
#pragma unroll
      for (int r = 0; r < kPlanes; ++r) *(uint4*)(place(0, q, i) + r * kPlane) = w[r];
    }
  }
  __device__ __forceinline__ void land() {      // !kVec: the row in the registers comes to its place
    land(s0, 0);
    if (kArrays > 1) land(s1, 1);
    if (kArrays > 2) land(s2, 2);
  }
  // The thread's values of piece i, which it has.
  __device__ __forceinline__ void values(int stage, int q, int i, float (&v)[8]) const {
    uint4 w[kPlanes];
    Eight<T> e;
#pragma unroll
    for (int r = 0; r < kPlanes; ++r) w[r] = *(const uint4*)(place(stage, q, i) + r * kPlane);
    memcpy(&e, w, sizeof w);
    e.widen_to(v);
  }
  __device__ __forceinline__ void meet() const {
    if (warps > 1) asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(warps * 32) : "memory");
  }
};

// The mean and the sum of squares around it meet in one exchange: a warp sums its columns, then their squares around its own mean, and of
// n columns with sum s and squares q the row takes q + n (s / n - mean)^2 (Chan, Golub and LeVeque, 1979).
template <class T, bool kVec, bool kFull, int kKeep, bool kResidual>
__global__ void __launch_bounds__(32 * kRowWarps, 1) k_layer_norm_rows(const __grid_constant__ NormArgs<T> a, int warps, int rows_per) {
  using Pipe = RowPipe<T, kVec, kFull, kKeep, kResidual ? 2 : 1>;
  extern __shared__ __align__(16) char norm_smem[];
  __shared__ float2 part[2][kRowWarps];
  Pipe pipe(norm_smem, warps, rows_per, a.rows, a.cols);
  const int lane = pipe.lane;
  launch_wait();
  launch_next();
  const uint32_t step = mask_step(a.mask);
  pipe.source(pipe.s0, a.x, a.ld_x);
  if (kResidual) pipe.source(pipe.s1, a.residual, a.ld_r);
  pipe.start(Pipe::kStages);
  constexpr bool kWeights = kKeep == 1 || (kVec && kKeep == 2);      // kept in registers
  float gamma[kWeights ? kKeep : 1][8] = {}, beta[kWeights ? kKeep : 1][8] = {};
  auto weights = [&](int i, float (&g)[8], float (&b)[8]) {
    if (a.gamma) load_cols<kVec>(a.gamma, pipe.base(i), lane, a.cols, g);
    if (a.beta) load_cols<kVec>(a.beta, pipe.base(i), lane, a.cols, b);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (!a.gamma) g[j] = 1.f;
      if (!a.beta) b[j] = 0.f;
    }
  };
  if constexpr (kWeights) {
#pragma unroll
    for (int i = 0; i < kKeep; ++i)
      if (pipe.on(i)) weights(i, gamma[i], beta[i]);
  }
  auto columns_of = [&](int warp) {      // of a row's warps
    int n = 0;
    for (int i = 0; i < kKeep; ++i) n += min(kWarpCols, max(0, a.cols - (i * warps + warp) * kWarpCols));
    return n;
  };
  const int n_own = columns_of(pipe.in_row), n_lane = lane < warps ? columns_of(lane) : 0;
  const float share_own = n_own ? 1.f / n_own : 0.f, share_lane = n_lane ? 1.f / n_lane : 0.f, share = 1.f / a.cols;
  const bool to_total = a.total != nullptr, masked = a.mask.limit != 0;
  T *y = a.y + pipe.first * a.ld_y, *total = a.total + (to_total ? pipe.first * a.ld_t : 0);
  const int64_t y_step = pipe.step * a.ld_y, total_step = pipe.step * a.ld_t;
  float v[kKeep][8], before[kKeep][8];
  int row = pipe.first, stage = 0;
  auto sums = [&](int k) {      // of row k, whose values come to v
    if constexpr (kVec) copies_wait<Pipe::kStages - 1>();
    else pipe.land();
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
      if (!pipe.works(i)) continue;
      pipe.values(stage, 0, i, v[i]);
      if (masked) drop_cols<kVec>(a.mask, step, (uint32_t)row, pipe.base(i), lane, v[i]);
      if constexpr (kResidual) {
        float r[8];
        pipe.values(stage, 1, i, r);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] += r[j];
      }
      sum += sum8(v[i]);
      if (to_total && pipe.on(i)) store_cols<T, kVec>(total, pipe.base(i), lane, a.cols, v[i]);
    }
    total += total_step;
    pipe.fetch();      // into the place of the row just read
    if constexpr (kVec) stage = stage + 1 == Pipe::kStages ? 0 : stage + 1;
    sum = warp_sum(sum);
    const float own = sum * share_own;
    float squares[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
      if (!pipe.works(i)) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = (kVec ? pipe.on(i) : col_of<kVec>(pipe.base(i), lane, j) < a.cols) ? v[i][j] - own : 0.f;
        squares[j & 1] = fmaf(d, d, squares[j & 1]);
      }
    }
    const float all = warp_sum(squares[0] + squares[1]);
    if (lane == 0) part[k & 1][pipe.group * warps + pipe.in_row] = make_float2(sum, all);
  };
  auto results = [&](int k, int row) {      // of row k, from `before`
    const float2 p = lane < warps ? part[k & 1][pipe.group * warps + lane] : make_float2(0.f, 0.f);
    const float mean = warp_sum(p.x) * share, off = p.x * share_lane - mean;
    const float rstd = inverse_root(warp_sum(fmaf(n_lane * off, off, p.y)) * share + a.eps);
    if (pipe.in_row == 0 && lane == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
      if (!pipe.works(i)) continue;
      if constexpr (!kWeights) weights(i, gamma[0], beta[0]);
      const float(&g)[8] = gamma[kWeights ? i : 0], (&b)[8] = beta[kWeights ? i : 0];
      float out[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) out[j] = fmaf((before[i][j] - mean) * rstd, g[j], b[j]);
      if (pipe.on(i)) store_cols<T, kVec>(y, pipe.base(i), lane, a.cols, out);
    }
    y += y_step;
  };
  if (!pipe.count) return;
  auto next = [&]() {
#pragma unroll
    for (int i = 0; i < kKeep; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) before[i][j] = v[i][j];
    row += pipe.step;
    pipe.meet();
  };
  sums(0);
  next();
#pragma unroll 1
  for (int k = 1; k < pipe.count; ++k) {
    sums(k);
    results(k - 1, row - pipe.step);
    next();
  }
  results(pipe.count - 1, row - pipe.step);
}

// Longer rows: a block takes one, each warp kLongKeep pieces of 256 columns in its registers; what is beyond is read again.  A thread adds eight
// values before they join its sum, so that of n columns n / 4096 follow one another there, not n / 512 (2^24 equal values: mean off by
// up to 6e-5 of itself, not 5e-4).
constexpr int kLongKeep = 4;
template <class T, bool kVec>
__global__ void __launch_bounds__(32 * kRowWarps) k_layer_norm_long(const __grid_constant__ NormArgs<T> a) {
  __shared__ float part[2][kRowWarps];
  constexpr int span = kRowWarps * kWarpCols;
  const int lane = threadIdx.x & 31, in_row = threadIdx.x >> 5;
  const int64_t row = blockIdx.x;
  launch_wait();
  launch_next();
  const uint32_t step = mask_step(a.mask);
  const T* x = a.x + row * a.ld_x;
  const T* res = a.residual ? a.residual + row * a.ld_r : nullptr;
  auto values = [&](const Eight<T>& ex, const Eight<T>& er, int base, float (&v)[8]) {
    ex.widen_to(v);
    if (a.mask.limit) drop_cols<kVec>(a.mask, step, (uint32_t)row, base, lane, v);
    if (res) {
      float q[8];
      er.widen_to(q);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += q[j];
    }
  };
  auto fetch = [&](int base, float (&v)[8]) {      // of a long row, what is not kept
    Eight<T> ex, er;
    load_cols<T, kVec>(x, base, lane, a.cols, ex);
    if (res) load_cols<T, kVec>(res, base, lane, a.cols, er);
    values(ex, er, base, v);
  };
  Eight<T> ex[kLongKeep], er[kLongKeep];
#pragma unroll
  for (int i = 0; i < kLongKeep; ++i) {
    const int base = i * span + in_row * kWarpCols;
    if (has_cols<kVec>(base, lane, a.cols)) {
      load_cols<T, kVec>(x, base, lane, a.cols, ex[i]);
      if (res) load_cols<T, kVec>(res, base, lane, a.cols, er[i]);
    }
  }
  const int rest = kLongKeep * span + in_row * kWarpCols;
  float v[kLongKeep][8], w[8], sum = 0.f;
#pragma unroll
  for (int i = 0; i < kLongKeep; ++i) {
    const int base = i * span + in_row * kWarpCols;
    if (!has_cols<kVec>(base, lane, a.cols)) break;
    values(ex[i], er[i], base, v[i]);
    sum += sum8(v[i]);
  }
  for (int base = rest; has_cols<kVec>(base, lane, a.cols); base += span) {
    fetch(base, w);
    sum += sum8(w);
  }
  const float mean = row_sum(sum, part[0]) / a.cols;
  float squares = 0.f;
  auto add_squares = [&](const float (&v)[8], int base) {
    float here = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = v[j] - mean;
      if (col_of<kVec>(base, lane, j) < a.cols) here = fmaf(d, d, here);
    }
    squares += here;
  };
#pragma unroll
  for (int i = 0; i < kLongKeep; ++i) {
    const int base = i * span + in_row * kWarpCols;
    if (!has_cols<kVec>(base, lane, a.cols)) break;
    add_squares(v[i], base);
  }
  for (int base = rest; has_cols<kVec>(base, lane, a.cols); base += span) {
    fetch(base, w);
    add_squares(w, base);
  }
  const float rstd = inverse_root(row_sum(squares, part[1]) / a.cols + a.eps);
  if (in_row == 0 && lane == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  auto finish = [&](const float (&v)[8], int base) {
    float g[8], b[8], y[8];
    if (a.gamma) load_cols<kVec>(a.gamma, base, lane, a.cols, g);
    if (a.beta) load_cols<kVec>(a.beta, base, lane, a.cols, b);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      y[j] = (v[j] - mean) * rstd;
      if (a.gamma) y[j] *= g[j];
      if (a.beta) y[j] += b[j];
    }
    if (a.total) store_cols<T, kVec>(a.total + row * a.ld_t, base, lane, a.cols, v);
    store_cols<T, kVec>(a.y + row * a.ld_y, base, lane, a.cols, y);
  };
#pragma unroll
  for (int i = 0; i < kLongKeep; ++i) {
    const int base = i * span + in_row * kWarpCols;
    if (!has_cols<kVec>(base, lane, a.cols)) break;
    finish(v[i], base);
  }
  for (int base = rest; has_cols<kVec>(base, lane, a.cols); base += span) {
    fetch(base, w);
    finish(w, base);
  }
}

template <class T>
struct NormBackArgs {
  const T *dy, *total, *dtotal;      // dtotal, dresidual, dx, gamma may be null
  T *dresidual, *dx;
  int64_t ld_dy, ld_t, ld_dt, ld_dr, ld_dx;
  const float *gamma, *mean, *rstd;
  int rows, cols;
  Mask mask;
};

template <class T, bool kVec>
__global__ void __launch_bounds__(32 * kRowWarps) k_layer_norm_back_long(const __grid_constant__ NormBackArgs<T> a) {
  __shared__ float part[2][kRowWarps];
  constexpr int span = kRowWarps * kWarpCols;
  const int lane = threadIdx.x & 31, in_row = threadIdx.x >> 5;
  const int64_t row = blockIdx.x;
  launch_wait();
  launch_next();
  const uint32_t step = mask_step(a.mask);
  const T *dy = a.dy + row * a.ld_dy, *total = a.total + row * a.ld_t;
  const float mean = a.mean[row], rstd = a.rstd[row];
  // g and h of 256 columns, zero past the end
  auto values = [&](const Eight<T>& ey, const Eight<T>& et, int base, float (&g)[8], float (&h)[8]) {
    ey.widen_to(g);
    et.widen_to(h);
    if (a.gamma) {
      float w[8];
      load_cols<kVec>(a.gamma, base, lane, a.cols, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] *= w[j];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = kVec || col_of<kVec>(base, lane, j) < a.cols ? (h[j] - mean) * rstd : 0.f;
  };
  auto fetch = [&](int base, float (&g)[8], float (&h)[8]) {
    Eight<T> ey, et;
    load_cols<T, kVec>(dy, base, lane, a.cols, ey);
    load_cols<T, kVec>(total, base, lane, a.cols, et);
    values(ey, et, base, g, h);
  };
  Eight<T> ey[kLongKeep], et[kLongKeep];
#pragma unroll
  for (int i = 0; i < kLongKeep; ++i) {
    const int base = i * span + in_row * kWarpCols;
    if (has_cols<kVec>(base, lane, a.cols)) {
      load_cols<T, kVec>(dy, base, lane, a.cols, ey[i]);
      load_cols<T, kVec>(total, base, lane, a.cols, et[i]);
    }
  }
  const int rest = kLongKeep * span + in_row * kWarpCols;
  float g[8], h[8], sum = 0.f, along = 0.f;
  auto add = [&]() {
    float here = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) here = fmaf(g[j], h[j], here);
    sum += sum8(g), along += here;
  };
#pragma unroll
  for (int i = 0; i < kLongKeep; ++i) {
    const int base = i * span + in_row * kWarpCols;
    if (!has_cols<kVec>(base, lane, a.cols)) break;
    values(ey[i], et[i], base, g, h);
    add();
  }
  for (int base = rest; has_cols<kVec>(base, lane, a.cols); base += span) {
    fetch(base, g, h);
    add();
  }
  sum = row_sum(sum, part[0]) / a.cols;
  along = row_sum(along, part[1]) / a.cols;
  auto finish = [&](int base) {
    float d[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) d[j] = (g[j] - sum - h[j] * along) * rstd;
    if (a.dtotal) {
      Eight<T> e;
      float q[8];
      load_cols<T, kVec>(a.dtotal + row * a.ld_dt, base, lane, a.cols, e);
      e.widen_to(q);
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j] += q[j];
    }
    if (a.dresidual) store_cols<T, kVec>(a.dresidual + row * a.ld_dr, base, lane, a.cols, d);
    if (a.dx) {
      drop_cols<kVec>(a.mask, step, (uint32_t)row, base, lane, d);
      store_cols<T, kVec>(a.dx + row * a.ld_dx, base, lane, a.cols, d);
    }
  };
#pragma unroll
  for (int i = 0; i < kLongKeep; ++i) {
    const int base = i * span + in_row * kWarpCols;
    if (!has_cols<kVec>(base, lane, a.cols)) break;
    values(ey[i], et[i], base, g, h);
    finish(base);
  }
  for (int base = rest; has_cols<kVec>(base, lane, a.cols); base += span) {
    fetch(base, g, h);
    finish(base);
  }
}

// The gradients of rows that fit the block.  A thread has the same columns of every row, so dgamma's and dbeta's sums stay in its
// registers; it reads a row in shared memory twice, for the row's two sums, then for the results.
template <class T, bool kVec, bool kFull, int kKeep, bool kMore>
__global__ void __launch_bounds__(32 * kRowWarps, 1) k_layer_norm_back_rows(const __grid_constant__ NormBackArgs<T> a, int warps, int rows_per, float* parts) {
  using Pipe = RowPipe<T, kVec, kFull, kKeep, kMore ? 3 : 2>;
  // With three stages a row's results wait until the next row's sums are on their way; with fewer its place is needed before.
  constexpr bool kLater = Pipe::kStages > 2;
  extern __shared__ __align__(16) char norm_smem[];
  __shared__ float2 part[2][kRowWarps];
  Pipe pipe(norm_smem, warps, rows_per, a.rows, a.cols);
  const int lane = pipe.lane;
  launch_wait();
  launch_next();
  const uint32_t step = mask_step(a.mask);
  pipe.source(pipe.s0, a.dy, a.ld_dy);
  pipe.source(pipe.s1, a.total, a.ld_t);
  if (kMore) pipe.source(pipe.s2, a.dtotal, a.ld_dt);
  pipe.start(kVec ? Pipe::kStages - 1 : 1);
  constexpr bool kWeights = kKeep == 1 || (kVec && kKeep == 2);      // kept in registers
  float gamma[kWeights ? kKeep : 1][8] = {};
  auto weights = [&](int i, float (&g)[8]) {
    if (a.gamma) load_cols<kVec>(a.gamma, pipe.base(i), lane, a.cols, g);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] = 1.f;
  };
  if constexpr (kWeights) {
#pragma unroll
    for (int i = 0; i < kKeep; ++i)
      if (pipe.on(i)) weights(i, gamma[i]);
  }
  float to_gamma[kKeep][8] = {}, to_beta[kKeep][8] = {};
  const float share = 1.f / a.cols;
  const bool to_residual = a.dresidual != nullptr, to_x = a.dx != nullptr;
  T *dresidual = a.dresidual + (to_residual ? pipe.first * a.ld_dr : 0), *dx = a.dx + (to_x ? pipe.first * a.ld_dx : 0);
  const int64_t dresidual_step = pipe.step * a.ld_dr, dx_step = pipe.step * a.ld_dx;
  int row = pipe.first, stage = 0;
  float next_mean = pipe.count ? a.mean[row] : 0.f, next_rstd = pipe.count ? a.rstd[row] : 0.f, mean = 0.f, rstd = 0.f, old_mean = 0.f, old_rstd = 0.f;
  // g and h of piece i of the row in `stage`; the mean is taken off first, so that h has two roundings however large the mean is
  auto read = [&](int stage, int i, float mean, float rstd, float (&g)[8], float (&h)[8]) {
    pipe.values(stage, 0, i, g);
    pipe.values(stage, 1, i, h);
    if (kVec && !pipe.on(i)) mean = 0.f;      // where there are no columns h is 0 like g, and not what -mean rstd may overflow to
#pragma unroll
    for (int j = 0; j < 8; j += 2) {      // in pairs, an instruction each: 227 us where single ones took 240 (gradients of 16384 x 8192, bfloat16)
      const float2 two = __fmul2_rn(__fadd2_rn(make_float2(h[j], h[j + 1]), make_float2(-mean, -mean)), make_float2(rstd, rstd));
      h[j] = two.x, h[j + 1] = two.y;
    }
    if (!kVec && !isfinite(mean * rstd))
#pragma unroll
      for (int j = 0; j < 8; ++j) h[j] = col_of<kVec>(pipe.base(i), lane, j) < a.cols ? h[j] : 0.f;
  };
  auto weigh = [&](int i, float (&g)[8]) {
    if constexpr (!kWeights) weights(i, gamma[0]);
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] *= gamma[kWeights ? i : 0][j];
  };
  auto results = [&](int k, int stage, int row, float mean, float rstd) {
    if (!to_residual && !to_x) return;
    const float2 p = lane < warps ? part[k & 1][pipe.group * warps + lane] : make_float2(0.f, 0.f);
    // rstd (g - mean(g) - h mean(g h)) = rstd g + (along h + level)
    const float along = -rstd * (warp_sum(p.y) * share), level = -rstd * (warp_sum(p.x) * share);
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
      if (!pipe.works(i)) continue;
      float g[8], d[8];
      read(stage, i, mean, rstd, g, d);
      weigh(i, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j] = fmaf(g[j], rstd, fmaf(d[j], along, level));
      if constexpr (kMore) {
        pipe.values(stage, 2, i, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] += g[j];
      }
      if (to_residual && pipe.on(i)) store_cols<T, kVec>(dresidual, pipe.base(i), lane, a.cols, d);
      if (to_x) {
        drop_cols<kVec>(a.mask, step, (uint32_t)row, pipe.base(i), lane, d);
        if (pipe.on(i)) store_cols<T, kVec>(dx, pipe.base(i), lane, a.cols, d);
      }
    }
    if (to_residual) dresidual += dresidual_step;
    if (to_x) dx += dx_step;
  };
  auto sums = [&](int k) {
    mean = next_mean, rstd = next_rstd;
    if (k + 1 < pipe.count) next_mean = a.mean[row + pipe.step], next_rstd = a.rstd[row + pipe.step];
    if constexpr (kVec) {
      if constexpr (!kLater) pipe.fetch();      // into the place of the row before
      copies_wait<kLater ? Pipe::kStages - 2 : Pipe::kStages - 1>();
    } else {
      pipe.land();
      pipe.fetch();
    }
    float sum[2] = {0.f, 0.f}, along[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
      if (!pipe.works(i)) continue;
      float g[8], h[8];
      read(stage, i, mean, rstd, g, h);
#pragma unroll
      for (int j = 0; j < 8; ++j) to_gamma[i][j] = fmaf(g[j], h[j], to_gamma[i][j]), to_beta[i][j] += g[j];
      weigh(i, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j & 1] += g[j], along[j & 1] = fmaf(g[j], h[j], along[j & 1]);
    }
    const float2 all = make_float2(warp_sum(sum[0] + sum[1]), warp_sum(along[0] + along[1]));
    if (lane == 0) part[k & 1][pipe.group * warps + pipe.in_row] = all;
  };
  auto next = [&]() {
    row += pipe.step;
    if constexpr (kVec) stage = stage + 1 == Pipe::kStages ? 0 : stage + 1;
  };
  if constexpr (kLater) {
    if (pipe.count) {
      sums(0);
      old_mean = mean, old_rstd = rstd;
      pipe.fetch();
      pipe.meet();
      next();
#pragma unroll 1
      for (int k = 1; k < pipe.count; ++k) {
        sums(k);
        results(k - 1, stage == 0 ? Pipe::kStages - 1 : stage - 1, row - pipe.step, old_mean, old_rstd);
        old_mean = mean, old_rstd = rstd;
        pipe.fetch();      // into the place of the row before
        pipe.meet();
        next();
      }
      results(pipe.count - 1, stage == 0 ? Pipe::kStages - 1 : stage - 1, row - pipe.step, old_mean, old_rstd);
    }
  } else {
#pragma unroll 1
    for (int k = 0; k < pipe.count; ++k) {
      sums(k);
      pipe.meet();
      results(k, stage, row, mean, rstd);
      next();
    }
  }
  if (!parts) return;
  // the groups' sums meet in the rows' places
  if constexpr (kVec) asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  float* met = (float*)norm_smem;
  const int width = warps * kWarpCols * kKeep;
#pragma unroll
  for (int i = 0; i < kKeep; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = col_of<kVec>(pipe.base(i), lane, j);
      met[(pipe.group * 2) * width + c] = to_gamma[i][j];
      met[(pipe.group * 2 + 1) * width + c] = to_beta[i][j];
    }
  __syncthreads();
  for (int k = 0; k < 2; ++k)
    for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
      float v = 0.f;
      for (int r = 0; r < rows_per; ++r) v += met[(r * 2 + k) * width + c];
      parts[((int64_t)blockIdx.x * 2 + k) * a.cols + c] = v;
    }
}

// Sums over the rows: 256 columns and a range of rows for each block, eight warps taking rows in turn; parts[blockIdx.y][2][cols].
template <class T, bool kVec>
__global__ void __launch_bounds__(256) k_norm_columns(const T* dy, int64_t ld_dy, const T* total, int64_t ld_t, const float* mean, const float* rstd, int rows, int cols,
                                                      int rows_per, float* parts) {
  __shared__ float sums[2][8][kWarpCols];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, base = blockIdx.x * kWarpCols;
  const int64_t r0 = (int64_t)blockIdx.y * rows_per;
  const int r1 = (int)min((int64_t)rows, r0 + rows_per);
  launch_wait();
  launch_next();
  float s[2][8] = {};
#pragma unroll 4
  for (int r = (int)r0 + warp; r < r1; r += 8) {
    Eight<T> ey, et;
    load_cols<T, kVec>(dy + r * ld_dy, base, lane, cols, ey);
    load_cols<T, kVec>(total + r * ld_t, base, lane, cols, et);
    const float m = mean[r], q = rstd[r];
    float y[8], t[8];
    ey.widen_to(y);
    et.widen_to(t);
#pragma unroll
    for (int j = 0; j < 8; ++j) s[0][j] = fmaf(y[j], (t[j] - m) * q, s[0][j]), s[1][j] += y[j];
  }
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[k][warp][j * 32 + lane] = s[k][j];
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * kWarpCols; i += 256) {
    const int k = i / kWarpCols, e = i % kWarpCols;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) v += sums[k][w][e];
    const int c = col_of<kVec>(base, e & 31, e >> 5);
    if (c < cols) parts[((int64_t)blockIdx.y * 2 + k) * cols + c] = v;
  }
}
// Adds the parts in binary64: 32 columns a block, 16 slices of the parts, each of whose loads are under way together, then the slices in
// their order.
constexpr int kJoinSlices = 16, kJoinTogether = 10;
__global__ void __launch_bounds__(32 * kJoinSlices) k_norm_join(const float* parts, int count, int cols, float* dgamma, float* dbeta) {
  __shared__ double sums[kJoinSlices][32];
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
  const int64_t i = (int64_t)blockIdx.x * 32 + lane, all = 2 * (int64_t)cols;
  launch_wait();
  launch_next();
  double s = 0.0;
  if (i < all) {
    for (int k = slice; k < count; k += kJoinSlices * kJoinTogether) {
      float v[kJoinTogether];
#pragma unroll
      for (int j = 0; j < kJoinTogether; ++j) v[j] = k + kJoinSlices * j < count ? parts[(k + kJoinSlices * j) * all + i] : 0.f;
#pragma unroll
      for (int j = 0; j < kJoinTogether; ++j) s += v[j];
    }
  }
  sums[slice][lane] = s;
  __syncthreads();
  if (slice || i >= all) return;
#pragma unroll
  for (int k = 1; k < kJoinSlices; ++k) s += sums[k][lane];
  if (i < cols) {
    if (dgamma) dgamma[i] = (float)s;
  } else if (dbeta) {
    dbeta[i - cols] = (float)s;
  }
}

}  // namespace mat
}  // namespace rtopk
