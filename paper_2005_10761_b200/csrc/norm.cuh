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
  uint32_t key0, key1, tag;  // tag: 2^31 + 2^16 site + worker, which no draw of the sampler has
  uint32_t step;
  const uint32_t* step_ptr;  // added to step when the kernel runs
};
__device__ __forceinline__ uint32_t mask_step(const Mask& m) { return m.step + (m.limit && m.step_ptr ? *m.step_ptr : 0u); }
// Bit j: column 8 group + j is kept.
__device__ __forceinline__ uint32_t kept8(const Mask& m, uint32_t step, uint32_t row, uint32_t group) {
  const uint4 x = philox4x32_10(group, row, m.tag, step, m.key0, m.key1);
  const uint32_t t = m.limit << 16;
  auto two = [&](uint32_t w) { return ((w << 16) >= t ? 1u : 0u) | (w >= t ? 2u : 0u); };
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
  const uint32_t own = kept8(m, step, row, (uint32_t)base / 8 + lane);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const bool kept = kVec ? own >> j & 1 : __shfl_sync(0xFFFFFFFFu, own, 4 * j + (lane >> 3)) >> (lane & 7) & 1;
    v[j] = kept ? v[j] * m.factor : 0.f;
  }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int k = 16; k; k >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, k);
  return v;
}
// The sum over a row's warps; `part` has a place for each warp of the block and is used once between two barriers.
template <int kWarps>
__device__ __forceinline__ float row_sum(float v, float* part) {
  v = warp_sum(v);
  if constexpr (kWarps > 1) {
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) part[warp] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) v += part[warp / kWarps * kWarps + i];
  }
  return v;
}

// ----------------------------------------------------------------------------- dropout
template <class T, bool kVec>
__global__ void __launch_bounds__(256) k_dropout(const T* x, int64_t ld_x, int64_t rows, int cols, int64_t band, const __grid_constant__ Mask mask, T* out, int64_t ld_out) {
  constexpr int kEach = 4;
  launch_wait();
  launch_next();
  const uint32_t step = mask_step(mask);
  const int lane = threadIdx.x & 31;
  const int64_t row0 = blockIdx.y * band;
  const int in_band = (int)min(band, rows - row0);
  if constexpr (kVec) {      // a thread: groups of eight columns, a block apart
    const uint32_t groups = (cols + 7) / 8, all = in_band * groups, first = blockIdx.x * (256u * kEach) + threadIdx.x;
    Eight<T> e[kEach];
    uint32_t r[kEach], g[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const uint32_t k = first + 256 * i;
      r[i] = k / groups, g[i] = k - r[i] * groups;
      if (k < all) e[i].load(x + (row0 + r[i]) * ld_x + g[i] * 8, cols - (int)g[i] * 8, true);
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (first + 256 * i >= all) break;
      float v[8];
      e[i].widen_to(v);
      const uint32_t kept = kept8(mask, step, (uint32_t)(row0 + r[i]), g[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = kept >> j & 1 ? v[j] * mask.factor : 0.f;
      store_cols<T, true>(out + (row0 + r[i]) * ld_out, g[i] * 8, 0, cols, v);
    }
  } else {                   // a warp: 256 columns of a row
    const uint32_t chunks = (cols + kWarpCols - 1) / kWarpCols, all = in_band * chunks;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const uint32_t k = blockIdx.x * (8u * kEach) + (threadIdx.x >> 5) + 8 * i;
      if (k >= all) break;
      const uint32_t r = k / chunks;
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
constexpr int kKeepChunks = 4;      // 256-column pieces of its row that a warp keeps in registers
template <int kWarps>
struct RowShape {
  static constexpr int kThreads = kWarps <= 8 ? 256 : 32 * kWarps, kRowsPer = kThreads / (32 * kWarps), kSpan = kWarps * kWarpCols;
};

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

template <class T, int kWarps, bool kVec>
__global__ void __launch_bounds__(RowShape<kWarps>::kThreads) k_layer_norm(const __grid_constant__ NormArgs<T> a) {
  using S = RowShape<kWarps>;
  __shared__ float part[2][S::kThreads / 32];
  const int lane = threadIdx.x & 31, in_row = (threadIdx.x >> 5) % kWarps;
  const int64_t at = (int64_t)blockIdx.x * S::kRowsPer + threadIdx.x / (32 * kWarps);
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
  Eight<T> ex[kKeepChunks], er[kKeepChunks];
#pragma unroll
  for (int i = 0; i < kKeepChunks; ++i) {
    const int base = i * S::kSpan + in_row * kWarpCols;
    if (base < a.cols) {
      load_cols<T, kVec>(x, base, lane, a.cols, ex[i]);
      if (res) load_cols<T, kVec>(res, base, lane, a.cols, er[i]);
    }
  }
  const int rest = kKeepChunks * S::kSpan + in_row * kWarpCols;
  float v[kKeepChunks][8], w[8], sum = 0.f;
#pragma unroll
  for (int i = 0; i < kKeepChunks; ++i) {
    const int base = i * S::kSpan + in_row * kWarpCols;
    if (base >= a.cols) break;
    values(ex[i], er[i], base, v[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += v[i][j];      // past the end they are zero
  }
  for (int base = rest; base < a.cols; base += S::kSpan) {
    fetch(base, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += w[j];
  }
  const float mean = row_sum<kWarps>(sum, part[0]) / a.cols;
  float squares = 0.f;
  auto add_squares = [&](const float (&v)[8], int base) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = v[j] - mean;
      if (col_of<kVec>(base, lane, j) < a.cols) squares = fmaf(d, d, squares);
    }
  };
#pragma unroll
  for (int i = 0; i < kKeepChunks; ++i) {
    const int base = i * S::kSpan + in_row * kWarpCols;
    if (base >= a.cols) break;
    add_squares(v[i], base);
  }
  for (int base = rest; base < a.cols; base += S::kSpan) {
    fetch(base, w);
    add_squares(w, base);
  }
  const float rstd = 1.f / sqrtf(row_sum<kWarps>(squares, part[1]) / a.cols + a.eps);
  if (!in) return;
  if (threadIdx.x % (32 * kWarps) == 0) {
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
  for (int i = 0; i < kKeepChunks; ++i) {
    const int base = i * S::kSpan + in_row * kWarpCols;
    if (base >= a.cols) break;
    finish(v[i], base);
  }
  for (int base = rest; base < a.cols; base += S::kSpan) {
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

template <class T, int kWarps, bool kVec>
__global__ void __launch_bounds__(RowShape<kWarps>::kThreads) k_layer_norm_back(const __grid_constant__ NormBackArgs<T> a) {
  using S = RowShape<kWarps>;
  __shared__ float part[2][S::kThreads / 32];
  const int lane = threadIdx.x & 31, in_row = (threadIdx.x >> 5) % kWarps;
  const int64_t at = (int64_t)blockIdx.x * S::kRowsPer + threadIdx.x / (32 * kWarps);
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
  Eight<T> ey[kKeepChunks], et[kKeepChunks];
#pragma unroll
  for (int i = 0; i < kKeepChunks; ++i) {
    const int base = i * S::kSpan + in_row * kWarpCols;
    if (base < a.cols) {
      load_cols<T, kVec>(dy, base, lane, a.cols, ey[i]);
      load_cols<T, kVec>(total, base, lane, a.cols, et[i]);
    }
  }
  const int rest = kKeepChunks * S::kSpan + in_row * kWarpCols;
  float g[8], h[8], sum = 0.f, along = 0.f;
  auto add = [&]() {
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += g[j], along = fmaf(g[j], h[j], along);
  };
#pragma unroll
  for (int i = 0; i < kKeepChunks; ++i) {
    const int base = i * S::kSpan + in_row * kWarpCols;
    if (base >= a.cols) break;
    values(ey[i], et[i], base, g, h);
    add();
  }
  for (int base = rest; base < a.cols; base += S::kSpan) {
    fetch(base, g, h);
    add();
  }
  sum = row_sum<kWarps>(sum, part[0]) / a.cols;
  along = row_sum<kWarps>(along, part[1]) / a.cols;
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
  for (int i = 0; i < kKeepChunks; ++i) {
    const int base = i * S::kSpan + in_row * kWarpCols;
    if (base >= a.cols) break;
    values(ey[i], et[i], base, g, h);
    finish(base);
  }
  for (int base = rest; base < a.cols; base += S::kSpan) {
    fetch(base, g, h);
    finish(base);
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
// Adds the parts in their order, in binary64.
__global__ void __launch_bounds__(256) k_norm_join(const float* parts, int count, int cols, float* dgamma, float* dbeta) {
  launch_wait();
  launch_next();
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= 2 * (int64_t)cols) return;
  double s = 0.0;
#pragma unroll 8
  for (int k = 0; k < count; ++k) s += parts[k * 2 * (int64_t)cols + i];
  if (i < cols) {
    if (dgamma) dgamma[i] = (float)s;
  } else if (dbeta) {
    dbeta[i - cols] = (float)s;
  }
}

}  // namespace mat
}  // namespace rtopk
