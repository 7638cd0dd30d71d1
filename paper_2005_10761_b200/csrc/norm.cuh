// Operators along the rows of a worker's activations: dropout from a counter-based generator, and layer normalisation with the
// dropout and the residual sum before it, forwards and backwards.
//
//   t = residual + D(x);   y = gamma (t - mean) rstd + beta                       mean and variance over the row
//   dt = rstd (g - mean(g) - h mean(g h)) + dtotal,  g = gamma dy, h = (t - mean) rstd;   dx = D(dt)
//   dgamma = sum over the rows of dy h,   dbeta = sum over the rows of dy
//
// All of it is bound by memory: a row is read once and kept in registers between its sums and its results.
#pragma once

#include "common.cuh"
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
// A warp takes 256 columns from `base`.  kVec: a thread has eight neighbours, in vectors; else every 32nd, so that loads and stores
// of rows without alignment are coalesced.
constexpr int kWarpCols = 256;
template <bool kVec>
__device__ __forceinline__ int col_of(int base, int lane, int j) { return kVec ? base + lane * 8 + j : base + j * 32 + lane; }

template <class T, bool kVec>
__device__ __forceinline__ void load_cols(const T* row, int base, int lane, int cols, Eight<T>& e) {
  if constexpr (kVec) {
    const int c = base + lane * 8;
    e.load(row + (c < cols ? c : 0), cols - c, true);
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
  Eight<float> e;
  load_cols<float, kVec>(row, base, lane, cols, e);
  e.widen_to(v);
}
__device__ __forceinline__ void narrow(float v, float& out) { out = v; }
__device__ __forceinline__ void narrow(float v, __nv_bfloat16& out) { out = __float2bfloat16_rn(v); }
template <class T, bool kVec>
__device__ __forceinline__ void store_cols(T* row, int base, int lane, int cols, const float (&v)[8]) {
  T q[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) narrow(v[j], q[j]);
  if (kVec && base + lane * 8 + 8 <= cols) {
    uint4* to = (uint4*)(row + base + lane * 8);
    uint4 w[sizeof(T) / 2];
    memcpy(w, q, sizeof w);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) to[i] = w[i];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = col_of<kVec>(base, lane, j);
      if (c < cols) row[c] = q[j];
    }
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

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int k = 16; k; k >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, k);
  return v;
}
// The sum over a row's `warps` warps; `part` has a place for each warp of the block and is used once between two barriers.
__device__ __forceinline__ float row_sum(float v, int warps, int group, float* part) {
  v = warp_sum(v);
  if (warps > 1) {
    const int lane = threadIdx.x & 31;
    if (lane == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = warp_sum(lane < warps ? part[group * warps + lane] : 0.f);
  }
  return v;
}

// ----------------------------------------------------------------------------- dropout
// Quotients of numbers below 2^31 by d: (k m / 2^32) / 2^shift with m = floor(2^(32 + shift) / d) + 1, 2^shift < d <= 2^(shift + 1); m is
// off by less than 1, which k times 2^-(32 + shift) keeps below 1 / d.
struct Divisor { uint32_t m, d; int shift; };
__device__ __forceinline__ uint32_t divide(uint32_t k, const Divisor& v) { return v.d == 1 ? k : __umulhi(k, v.m) >> v.shift; }

template <class T, bool kVec>
__global__ void __launch_bounds__(256) k_dropout(const T* x, int64_t ld_x, int64_t rows, int cols, int64_t band, const Divisor units, const __grid_constant__ Mask mask, T* out, int64_t ld_out) {
  constexpr int kEach = 4;
  launch_wait();
  launch_next();
  const uint32_t step = mask_step(mask);
  const int lane = threadIdx.x & 31;
  const int64_t row0 = blockIdx.y * band;
  const int in_band = (int)min(band, rows - row0);
  if constexpr (kVec) {      // a thread: groups of eight columns, a block apart
    const uint32_t groups = units.d, all = in_band * groups, first = blockIdx.x * (256u * kEach) + threadIdx.x;
    Eight<T> e[kEach];
    uint32_t r[kEach], g[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const uint32_t k = first + 256 * i;
      r[i] = divide(k, units), g[i] = k - r[i] * groups;
      if (k < all) e[i].load(x + (row0 + r[i]) * ld_x + g[i] * 8, cols - (int)g[i] * 8, true);
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (first + 256 * i >= all) break;
      float v[8];
      e[i].widen_to(v);
      drop8(mask, mask_words(mask, step, (uint32_t)(row0 + r[i]), g[i]), v);
      store_cols<T, true>(out + (row0 + r[i]) * ld_out, g[i] * 8, 0, cols, v);
    }
  } else {                   // a warp: 256 columns of a row
    const uint32_t chunks = units.d, all = in_band * chunks;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const uint32_t k = blockIdx.x * (8u * kEach) + (threadIdx.x >> 5) + 8 * i;
      if (k >= all) break;
      const uint32_t r = divide(k, units);
      const int base = (int)(k - r * chunks) * kWarpCols;
      Eight<T> e;
      load_cols<T, false>(x + (row0 + r) * ld_x, base, lane, cols, e);
      float v[8];
      e.widen_to(v);
      drop_cols<false>(mask, step, (uint32_t)(row0 + r), base, lane, v);
      store_cols<T, false>(out + (row0 + r) * ld_out, base, lane, cols, v);
    }
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

// Rows that fit the block are taken in turn: one block per SM, `rows_per` rows of it at a time with `warps` warps each, kKeep pieces of 256 columns
// a warp.  What a thread needs of the next rows is on its way to its own place in shared memory (kVec: asynchronous copies, `stages`
// rows deep; else by way of registers), so that no barrier stops the stream of reads.
//
// The bound is memory as long as the instructions keep up: 16 columns a thread, so that a row's sums, addresses and statistics are shared
// by 16; numbers of the mask compared two at a time.
constexpr int kRowWarps = 16, kRowSmem = 216 * 1024;
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {      // the rest of 16 becomes zero
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait(int left) {
  if (left == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else if (left == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else asm volatile("cp.async.wait_group 3;" ::: "memory");
}

template <class T, bool kVec, int kKeep, int kArrays>
struct RowPipe {
  static constexpr int kPlanes = sizeof(T) / 2;      // a thread's eight values lie in pieces of 16 bytes, each thread's next to the others'
  int warps, group, in_row, lane, stages, arrays, plane, cols;
  int sets;                    // of rows, of this block
  int64_t first, step, rows;   // the thread's row of a set is first + set * step
  char* mine;
  struct Source {
    const T* p;      // of the next row to be read
    int64_t step;
    Eight<T> next[kVec ? 1 : kKeep];
  } s0, s1, s2;

  __device__ __forceinline__ RowPipe(char* smem, int warps, int rows_per, int stages, int64_t rows, int cols) : warps(warps), stages(stages), cols(cols), rows(rows) {
    lane = threadIdx.x & 31;
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0);
    group = warp / warps, in_row = warp - group * warps;
    plane = warps * 512;
    arrays = 0;
    first = (int64_t)blockIdx.x * rows_per + group, step = (int64_t)gridDim.x * rows_per;
    const int64_t all = (rows + rows_per - 1) / rows_per;
    sets = blockIdx.x < all ? (int)((all - 1 - blockIdx.x) / gridDim.x) + 1 : 0;
    mine = smem;
  }
  __device__ __forceinline__ void add(Source& s, const T* p, int64_t ld) {      // in the order of s0, s1, s2
    if (!p) return;
    s.p = p + first * ld + (kVec ? base(0) + lane * 8 : 0), s.step = ld * step;
    ++arrays;
  }
  __device__ __forceinline__ void start() {
    mine += group * stages * arrays * kKeep * kPlanes * plane + (in_row * 32 + lane) * 16;
    if constexpr (kVec)
      for (int k = 0; k < stages - 1; ++k) fetch(k, k);
    else fetch(0, 0);
  }
  __device__ __forceinline__ int base(int i) const { return (i * warps + in_row) * kWarpCols; }
  __device__ __forceinline__ char* place(int stage, int q, int i) const { return mine + ((stage * arrays + q) * kKeep + i) * kPlanes * plane; }
  __device__ __forceinline__ void fetch(Source& s, int q, int stage) {
    const uint32_t to = smem_addr(place(stage, q, 0));
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
      if constexpr (kVec) {
        const int left = (cols - base(i) - lane * 8) * (int)sizeof(T);
#pragma unroll
        for (int r = 0; r < kPlanes; ++r)
          if (left > 16 * r) copy16(to + (i * kPlanes + r) * plane, (const char*)(s.p + i * warps * kWarpCols) + 16 * r, min(16, left - 16 * r));
      } else {
        load_cols<T, false>(s.p, base(i), lane, cols, s.next[i]);
      }
    }
    s.p += s.step;
  }
  __device__ __forceinline__ void fetch(int k, int stage) {      // called for k = 0, 1, 2, ..
    if (k < sets && first + k * step < rows) {
      fetch(s0, 0, stage);
      if (arrays > 1) fetch(s1, 1, stage);
      if (kArrays > 2 && arrays > 2) fetch(s2, 2, stage);
    }
    if constexpr (kVec) copies_commit();
  }
  __device__ __forceinline__ void land(const Source& s, int q) {
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
      uint4 w[kPlanes];
      memcpy(w, &s.next[i], sizeof w);
#pragma unroll
      for (int r = 0; r < kPlanes; ++r) *(uint4*)(place(0, q, i) + r * plane) = w[r];
    }
  }
  // Brings row k's values in and the row that follows on its way.
  __device__ __forceinline__ void advance(int k, int stage) {
    if constexpr (kVec) {
      fetch(k + stages - 1, stage == 0 ? stages - 1 : stage - 1);
      copies_wait(stages - 1);
    } else {
      if (first + k * step < rows) {
        land(s0, 0);
        if (arrays > 1) land(s1, 1);
        if (kArrays > 2 && arrays > 2) land(s2, 2);
      }
      fetch(k + 1, 0);
    }
  }
  // The thread's values of piece i; pieces that end inside hold zeros beyond.
  __device__ __forceinline__ void values(int stage, int q, int i, float (&v)[8]) const {
    uint4 w[kPlanes];
    Eight<T> e;
#pragma unroll
    for (int r = 0; r < kPlanes; ++r) w[r] = *(const uint4*)(place(stage, q, i) + r * plane);
    memcpy(&e, w, sizeof w);
    e.widen_to(v);
  }
  __device__ __forceinline__ void zero() {      // places that no copy fills
    if constexpr (kVec) {
      for (int s = 0; s < stages; ++s)
        for (int q = 0; q < arrays; ++q)
#pragma unroll
          for (int i = 0; i < kKeep; ++i)
#pragma unroll
            for (int r = 0; r < kPlanes; ++r)
              if ((cols - base(i) - lane * 8) * (int)sizeof(T) <= 16 * r) *(uint4*)(place(s, q, i) + r * plane) = make_uint4(0u, 0u, 0u, 0u);
    }
  }
  // Sums over the row's warps; `part` has a place for each warp and is used again after another call's barrier.
  __device__ __forceinline__ void meet() const { asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(warps * 32) : "memory"); }
  __device__ __forceinline__ float sum(float v, float* part) const {
    v = warp_sum(v);
    if (warps == 1) return v;
    if (lane == 0) part[group * warps + in_row] = v;
    meet();
    return warp_sum(lane < warps ? part[group * warps + lane] : 0.f);
  }
  __device__ __forceinline__ float2 sum(float2 v, float2* part) const {
    v = make_float2(warp_sum(v.x), warp_sum(v.y));
    if (warps == 1) return v;
    if (lane == 0) part[group * warps + in_row] = v;
    meet();
    v = lane < warps ? part[group * warps + lane] : make_float2(0.f, 0.f);
    return make_float2(warp_sum(v.x), warp_sum(v.y));
  }
};

template <class T, bool kVec, int kKeep>
__global__ void __launch_bounds__(32 * kRowWarps, 1) k_layer_norm_rows(const __grid_constant__ NormArgs<T> a, int warps, int rows_per, int stages) {
  extern __shared__ __align__(16) char norm_smem[];
  __shared__ float part[4][kRowWarps];
  RowPipe<T, kVec, kKeep, 2> pipe(norm_smem, warps, rows_per, stages, a.rows, a.cols);
  const int lane = pipe.lane;
  launch_wait();
  launch_next();
  const uint32_t step = mask_step(a.mask);
  pipe.add(pipe.s0, a.x, a.ld_x);
  pipe.add(pipe.s1, a.residual, a.ld_r);
  pipe.start();
  pipe.zero();
  constexpr bool kWeights = kKeep <= 2;      // kept in registers
  float gamma[kWeights ? kKeep : 1][8], beta[kWeights ? kKeep : 1][8];
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
      if (pipe.base(i) < a.cols) weights(i, gamma[i], beta[i]);
  }
  const float share = 1.f / a.cols;
  int stage = 0;
#pragma unroll 1
  for (int k = 0; k < pipe.sets; ++k) {
    const int64_t row = pipe.first + k * pipe.step;
    pipe.advance(k, stage);
    if (row >= a.rows) break;      // the same for all of a row's warps; only in the block's last set
    float v[kKeep][8], sum = 0.f;
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
      if (pipe.base(i) >= a.cols) break;
      pipe.values(stage, 0, i, v[i]);
      if (a.mask.limit) drop_cols<kVec>(a.mask, step, (uint32_t)row, pipe.base(i), lane, v[i]);
      if (a.residual) {
        float r[8];
        pipe.values(stage, 1, i, r);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] += r[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += v[i][j];
    }
    const float mean = pipe.sum(sum, part[k & 1]) * share;
    float squares = 0.f;
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
      const int base = pipe.base(i);
      if (base >= a.cols) break;
      if (base + kWarpCols <= a.cols) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float d = v[i][j] - mean;
          squares = fmaf(d, d, squares);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float d = v[i][j] - mean;
          if (col_of<kVec>(base, lane, j) < a.cols) squares = fmaf(d, d, squares);
        }
      }
    }
    const float rstd = 1.f / sqrtf(pipe.sum(squares, part[2 + (k & 1)]) * share + a.eps);
    if (pipe.in_row == 0 && lane == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
      const int base = pipe.base(i);
      if (base >= a.cols) break;
      if (a.total) store_cols<T, kVec>(a.total + row * a.ld_t, base, lane, a.cols, v[i]);
      if constexpr (!kWeights) weights(i, gamma[0], beta[0]);
      const float(&g)[8] = gamma[kWeights ? i : 0], (&b)[8] = beta[kWeights ? i : 0];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = fmaf((v[i][j] - mean) * rstd, g[j], b[j]);
      store_cols<T, kVec>(a.y + row * a.ld_y, base, lane, a.cols, v[i]);
    }
    if constexpr (kVec) stage = stage + 1 == stages ? 0 : stage + 1;
  }
}

// Longer rows: `warps` warps take a row, each kKeep pieces of 256 columns in its registers; what is beyond is read again.
template <class T, bool kVec, int kKeep>
__global__ void __launch_bounds__(512) k_layer_norm(const __grid_constant__ NormArgs<T> a, int warps, int rows_per) {
  __shared__ float part[2][16];
  const int lane = threadIdx.x & 31, group = (threadIdx.x >> 5) / warps, in_row = (threadIdx.x >> 5) - group * warps, span = warps * kWarpCols;
  const int64_t at = (int64_t)blockIdx.x * rows_per + group;
  const bool in = at < a.rows;
  const int64_t row = in ? at : a.rows - 1;
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
  Eight<T> ex[kKeep], er[kKeep];
#pragma unroll
  for (int i = 0; i < kKeep; ++i) {
    const int base = i * span + in_row * kWarpCols;
    if (base < a.cols) {
      load_cols<T, kVec>(x, base, lane, a.cols, ex[i]);
      if (res) load_cols<T, kVec>(res, base, lane, a.cols, er[i]);
    }
  }
  const int rest = kKeep * span + in_row * kWarpCols;
  float v[kKeep][8], w[8], sum = 0.f;
#pragma unroll
  for (int i = 0; i < kKeep; ++i) {
    const int base = i * span + in_row * kWarpCols;
    if (base >= a.cols) break;
    values(ex[i], er[i], base, v[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += v[i][j];      // past the end they are zero
  }
  for (int base = rest; base < a.cols; base += span) {
    fetch(base, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += w[j];
  }
  const float mean = row_sum(sum, warps, group, part[0]) / a.cols;
  float squares = 0.f;
  auto add_squares = [&](const float (&v)[8], int base) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = v[j] - mean;
      if (col_of<kVec>(base, lane, j) < a.cols) squares = fmaf(d, d, squares);
    }
  };
#pragma unroll
  for (int i = 0; i < kKeep; ++i) {
    const int base = i * span + in_row * kWarpCols;
    if (base >= a.cols) break;
    add_squares(v[i], base);
  }
  for (int base = rest; base < a.cols; base += span) {
    fetch(base, w);
    add_squares(w, base);
  }
  const float rstd = 1.f / sqrtf(row_sum(squares, warps, group, part[1]) / a.cols + a.eps);
  if (!in) return;
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
  for (int i = 0; i < kKeep; ++i) {
    const int base = i * span + in_row * kWarpCols;
    if (base >= a.cols) break;
    finish(v[i], base);
  }
  for (int base = rest; base < a.cols; base += span) {
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

template <class T, bool kVec, int kKeep>
__global__ void __launch_bounds__(512) k_layer_norm_back(const __grid_constant__ NormBackArgs<T> a, int warps, int rows_per) {
  __shared__ float part[2][16];
  const int lane = threadIdx.x & 31, group = (threadIdx.x >> 5) / warps, in_row = (threadIdx.x >> 5) - group * warps, span = warps * kWarpCols;
  const int64_t at = (int64_t)blockIdx.x * rows_per + group;
  const bool in = at < a.rows;
  const int64_t row = in ? at : a.rows - 1;
  launch_wait();
  launch_next();
  const uint32_t step = mask_step(a.mask);
  const T *dy = a.dy + row * a.ld_dy, *total = a.total + row * a.ld_t;
  const float mean = a.mean[row], rstd = a.rstd[row];
  // g and h of 256 columns; past the end g is zero
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
    for (int j = 0; j < 8; ++j) h[j] = (h[j] - mean) * rstd;
  };
  auto fetch = [&](int base, float (&g)[8], float (&h)[8]) {
    Eight<T> ey, et;
    load_cols<T, kVec>(dy, base, lane, a.cols, ey);
    load_cols<T, kVec>(total, base, lane, a.cols, et);
    values(ey, et, base, g, h);
  };
  Eight<T> ey[kKeep], et[kKeep];
#pragma unroll
  for (int i = 0; i < kKeep; ++i) {
    const int base = i * span + in_row * kWarpCols;
    if (base < a.cols) {
      load_cols<T, kVec>(dy, base, lane, a.cols, ey[i]);
      load_cols<T, kVec>(total, base, lane, a.cols, et[i]);
    }
  }
  const int rest = kKeep * span + in_row * kWarpCols;
  float g[8], h[8], sum = 0.f, along = 0.f;
  auto add = [&]() {
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += g[j], along = fmaf(g[j], h[j], along);
  };
#pragma unroll
  for (int i = 0; i < kKeep; ++i) {
    const int base = i * span + in_row * kWarpCols;
    if (base >= a.cols) break;
    values(ey[i], et[i], base, g, h);
    add();
  }
  for (int base = rest; base < a.cols; base += span) {
    fetch(base, g, h);
    add();
  }
  sum = row_sum(sum, warps, group, part[0]) / a.cols;
  along = row_sum(along, warps, group, part[1]) / a.cols;
  if (!in) return;
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
  for (int i = 0; i < kKeep; ++i) {
    const int base = i * span + in_row * kWarpCols;
    if (base >= a.cols) break;
    values(ey[i], et[i], base, g, h);
    finish(base);
  }
  for (int base = rest; base < a.cols; base += span) {
    fetch(base, g, h);
    finish(base);
  }
}

// The gradients of rows that fit the block.  A thread has the same columns of every row, so dgamma's and dbeta's sums stay in its
// registers; it reads a row in shared memory twice, for the row's two sums, then for the results.  One barrier a row.
template <class T, bool kVec, int kKeep>
__global__ void __launch_bounds__(32 * kRowWarps, 1) k_layer_norm_back_rows(const __grid_constant__ NormBackArgs<T> a, int warps, int rows_per, int stages, float* parts) {
  extern __shared__ __align__(16) char norm_smem[];
  __shared__ float2 part[2][kRowWarps];
  RowPipe<T, kVec, kKeep, 3> pipe(norm_smem, warps, rows_per, stages, a.rows, a.cols);
  const int lane = pipe.lane;
  launch_wait();
  launch_next();
  const uint32_t step = mask_step(a.mask);
  pipe.add(pipe.s0, a.dy, a.ld_dy);
  pipe.add(pipe.s1, a.total, a.ld_t);
  pipe.add(pipe.s2, a.dtotal, a.ld_dt);
  pipe.start();
  pipe.zero();
  constexpr bool kWeights = kKeep <= 2;      // kept in registers
  float gamma[kWeights ? kKeep : 1][8];
  auto weights = [&](int i, float (&g)[8]) {
    if (a.gamma) load_cols<kVec>(a.gamma, pipe.base(i), lane, a.cols, g);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] = 1.f;
  };
  if constexpr (kWeights) {
#pragma unroll
    for (int i = 0; i < kKeep; ++i)
      if (pipe.base(i) < a.cols) weights(i, gamma[i]);
  }
  float to_gamma[kKeep][8] = {}, to_beta[kKeep][8] = {};
  auto stat = [&](const float* p, int k) {
    const int64_t row = pipe.first + k * pipe.step;
    return k < pipe.sets && row < a.rows ? p[row] : 0.f;
  };
  float next_mean = stat(a.mean, 0), next_rstd = stat(a.rstd, 0);
  const float share = 1.f / a.cols;
  int stage = 0;
#pragma unroll 1
  for (int k = 0; k < pipe.sets; ++k) {
    const int64_t row = pipe.first + k * pipe.step;
    pipe.advance(k, stage);
    if (row >= a.rows) break;      // the same for all of a row's warps; only in the block's last set
    const float rstd = next_rstd, shift = -next_mean * rstd;
    next_mean = stat(a.mean, k + 1), next_rstd = stat(a.rstd, k + 1);
    float2 sums = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
      if (pipe.base(i) >= a.cols) break;
      float g[8], h[8];
      pipe.values(stage, 0, i, g);
      pipe.values(stage, 1, i, h);
      if constexpr (!kWeights) weights(i, gamma[0]);
      const float(&w)[8] = gamma[kWeights ? i : 0];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        h[j] = fmaf(h[j], rstd, shift);
        to_gamma[i][j] = fmaf(g[j], h[j], to_gamma[i][j]), to_beta[i][j] += g[j];
        g[j] *= w[j];
        sums.x += g[j], sums.y = fmaf(g[j], h[j], sums.y);
      }
    }
    if (a.dresidual || a.dx) {
      sums = pipe.sum(sums, part[k & 1]);
      // rstd (g - mean(g) - h mean(g h)) = rstd g + (along h + level)
      const float along = -rstd * (sums.y * share), level = -rstd * (sums.x * share);
#pragma unroll
      for (int i = 0; i < kKeep; ++i) {
        const int base = pipe.base(i);
        if (base >= a.cols) break;
        float g[8], d[8];
        pipe.values(stage, 0, i, g);
        pipe.values(stage, 1, i, d);
        if constexpr (!kWeights) weights(i, gamma[0]);
        const float(&w)[8] = gamma[kWeights ? i : 0];
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = fmaf(g[j] * w[j], rstd, fmaf(fmaf(d[j], rstd, shift), along, level));
        if (a.dtotal) {
          pipe.values(stage, 2, i, g);
#pragma unroll
          for (int j = 0; j < 8; ++j) d[j] += g[j];
        }
        if (a.dresidual) store_cols<T, kVec>(a.dresidual + row * a.ld_dr, base, lane, a.cols, d);
        if (a.dx) {
          drop_cols<kVec>(a.mask, step, (uint32_t)row, base, lane, d);
          store_cols<T, kVec>(a.dx + row * a.ld_dx, base, lane, a.cols, d);
        }
      }
    }
    if constexpr (kVec) stage = stage + 1 == stages ? 0 : stage + 1;
  }
  if (!parts) return;
  // the groups' sums meet in the rows' places
  if constexpr (kVec) asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  float* sums = (float*)norm_smem;
  const int width = warps * kWarpCols * kKeep;
#pragma unroll
  for (int i = 0; i < kKeep; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = col_of<kVec>(pipe.base(i), lane, j);
      sums[(pipe.group * 2) * width + c] = to_gamma[i][j];
      sums[(pipe.group * 2 + 1) * width + c] = to_beta[i][j];
    }
  __syncthreads();
  for (int k = 0; k < 2; ++k)
    for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
      float v = 0.f;
      for (int r = 0; r < rows_per; ++r) v += sums[(r * 2 + k) * width + c];
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
// Adds the parts in binary64: 32 columns a block, eight slices of the parts in turn, then the slices in their order.
__global__ void __launch_bounds__(256) k_norm_join(const float* parts, int count, int cols, float* dgamma, float* dbeta) {
  __shared__ double sums[8][32];
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
  const int64_t i = (int64_t)blockIdx.x * 32 + lane, all = 2 * (int64_t)cols;
  launch_wait();
  launch_next();
  double s = 0.0;
  if (i < all) {
#pragma unroll 4
    for (int k = slice; k < count; k += 8) s += parts[k * all + i];
  }
  sums[slice][lane] = s;
  __syncthreads();
  if (slice || i >= all) return;
#pragma unroll
  for (int k = 1; k < 8; ++k) s += sums[k][lane];
  if (i < cols) {
    if (dgamma) dgamma[i] = (float)s;
  } else if (dbeta) {
    dbeta[i - cols] = (float)s;
  }
}

}  // namespace mat
}  // namespace rtopk
