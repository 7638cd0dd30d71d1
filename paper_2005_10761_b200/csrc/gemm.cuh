// The tensor-core product of the matrix operators: D[lane][col] = sum_k P[lane][k] Q[col][k], 16-bit floating point
// with 32-bit sums or 8-bit integers with 32-bit integer sums, and what is done with D before it leaves the SM.
//
// One persistent block per SM, ten warps: one thread feeds a ring of shared-memory stages by TMA, one thread issues
// the products (128 x kCols tiles, the accumulators twice in tensor memory), eight warps turn finished tiles into
// results while the next tile is being multiplied.  D is always laid out so that the 32 lanes of a warp are
// neighbours in the result's rows: the stores are coalesced without a pass through shared memory.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tensorcore.cuh"

namespace rtopk {
namespace mat {

constexpr int kEpiWarps = 8;                // two for each quarter of the accumulator's lanes, taking its column chunks in turn
constexpr int kGemmThreads = 64 + 32 * kEpiWarps;
constexpr int kLanes = 128;                 // rows of an accumulator tile (tensor-memory lanes)
constexpr int kDepthBytes = 128;            // bytes of the contraction index per stage and row: one swizzle row
constexpr int kSmemLimit = 227 * 1024;
constexpr int kSmemMisc = 1024 + 1024;      // alignment slack, barriers

// Scales that keep 16-bit entries away from the subnormal range: X is held times 32 and its Gram matrix and the
// polynomial of it times 1024.  ||X||_F = 1 at the start, so an entry of a 10000 x 1500 X is about 2.6e-4; afterwards
// singular values stay below about 1.3, so nothing comes near the largest 16-bit number.
constexpr float kXScale = 32.f, kAScale = 1024.f, kLoScale = 2048.f;

enum Epi : int {
  EPI_GRAM = 0,    // A = X X^T: entries off the diagonal in 16 bits, the diagonal (from the unrounded X) in 32
  EPI_POLY = 1,    // a + b A + c A^2, in the same form
  EPI_APPLY = 2,   // X <- (that) X, as high and low halves
  EPI_OUT = 3,     // the last X, into the caller's matrix
  EPI_UPDATE = 4,  // the last X, into the caller's weights
  EPI_CODED = 5    // 8-bit codes: times the two scales
};

struct Gemm {
  int lanes, cols, depth;    // D is lanes x cols; depth in elements
  int batch, tiles_l, tiles_c, tiles;   // tiles per batch entry
  int tri;                   // only tiles that reach the upper triangle (col >= lane)
  uint32_t* error;
  // epilogue operands
  const __half* o;           // POLY: A off the diagonal; APPLY / OUT / UPDATE: high halves of X
  __half* lo;                // APPLY / OUT / UPDATE: low halves of X (APPLY: replaced in place)
  __half* h;                 // 16-bit result
  int64_t ld, stride;        // of o, lo, h
  const float* d_in;         // diagonal of the left operand [batch][cols]
  float* d_out;
  int64_t d_stride;
  float* row_sums;           // squares of X along 32 neighbours of a row: [batch][slots][d_stride]; APPLY writes, GRAM reads
  int slots;
  float a, b, c;
  void* out;                 // OUT, UPDATE, CODED
  int64_t out_col, out_lane, out_batch;     // element strides of the result by col, lane and batch entry
  int out_bf16;
  float keep, rate;          // UPDATE: w <- keep w - rate x
  const float* scale_col;    // CODED
  const float* scale_lane;   // CODED; null: 1
};

struct Tile { int l, c, z; };

template <int kCols>
__device__ __forceinline__ Tile tile_at(const Gemm& g, int t) {
  Tile r;
  r.z = t / g.tiles;
  int k = t - r.z * g.tiles;
  if (!g.tri) {
    r.c = k / g.tiles_l;
    r.l = k - r.c * g.tiles_l;
    return r;
  }
  // column tile c reaches the lane tiles 0 .. ((c + 1) kCols - 1) / 128
  for (r.c = 0;; ++r.c) {
    const int n = min(g.tiles_l, ((r.c + 1) * kCols - 1) / kLanes + 1);
    if (k < n) break;
    k -= n;
  }
  r.l = k;
  return r;
}

__device__ __forceinline__ __half to_half(float v) { return __float2half_rn(v); }

// Eight neighbours along a row of the 16-bit result.
__device__ __forceinline__ void store_half8(__half* p, const float* v) {
  __half2 h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
  *reinterpret_cast<uint4*>(p) = *reinterpret_cast<uint4*>(h);
}

// The entry of the Gram matrix's diagonal that belongs to `lane`, from the partial sums of squares; taken before the
// tile's products are waited for.
__device__ __forceinline__ float gram_diagonal(const Gemm& g, int z, int lane) {
  if (lane >= g.lanes) return 0.f;
  const float* sums = g.row_sums + (int64_t)z * g.slots * g.d_stride + lane;
  float d = 0.f;
#pragma unroll 16
  for (int i = 0; i < g.slots; ++i) d += sums[i * g.d_stride];
  return d * (1.f / kAScale);
}

// 32 entries of one lane, columns col0 .. (those past the edge read the last one): all loads are under way before the
// first is used.
__device__ __forceinline__ void load_column(const __half* p, int col0, int ncol, int64_t ld, __half (&v)[32]) {
  p += col0 * ld;
#pragma unroll
  for (int c = 0; c < 32; ++c) v[c] = p[min(c, ncol - 1) * ld];
}

// 32 columns (col0 ..) of lane `lane` of one tile.
template <int kEpi>
__device__ __forceinline__ void epilogue(const Gemm& g, int z, int lane, int col0, float diag, const uint32_t (&acc)[32]) {
  const int ncol = min(32, g.cols - col0);
  if (kEpi == EPI_GRAM || kEpi == EPI_POLY) {
    // Symmetric result: a 128-wide block of columns left of this lane's block is the mirror image of another tile.
    const int lb = lane / kLanes, cb = col0 / kLanes;
    if (cb < lb) return;
    const bool in = lane < g.lanes;
    lane = min(lane, g.lanes - 1);
    constexpr uint32_t active = 0xFFFFFFFFu;
    const float* d_in = g.d_in + z * g.d_stride;
    const __half* o = g.o + z * g.stride;
    __half* h = g.h + z * g.stride;
    float v[32];
    if (kEpi == EPI_GRAM) {
#pragma unroll
      for (int c = 0; c < 32; ++c) v[c] = __uint_as_float(acc[c]);
    } else {
      const float dl = d_in[lane], dc = d_in[col0 + min(threadIdx.x & 31, ncol - 1)];
      __half oc[32];
      load_column(o + lane, col0, ncol, g.ld, oc);
#pragma unroll
      for (int c = 0; c < 32; ++c) {
        const float d = __shfl_sync(active, dc, c);
        v[c] = c < ncol ? g.c * (__uint_as_float(acc[c]) * (1.f / kAScale)) + (g.b + g.c * (dl + d)) * __half2float(oc[c]) : 0.f;
      }
    }
    if (in && lane >= col0 && lane < col0 + ncol) {
      float q = 0.f;
#pragma unroll
      for (int c = 0; c < 32; ++c)
        if (lane == col0 + c) {
          q = __uint_as_float(acc[c]) * (1.f / kAScale);
          v[c] = 0.f;
        }
      if (kEpi == EPI_POLY) {
        const float x = d_in[lane];
        diag = g.a + g.b * x + g.c * (x * x + q * (1.f / kAScale));
      }
      g.d_out[z * g.d_stride + lane] = diag;
    }
    if (!in) return;
    // row `lane`, columns col0 ..: the row stride is a multiple of 8, so the padding takes whole vectors
    __half* row = h + (int64_t)lane * g.ld + col0;
#pragma unroll
    for (int c = 0; c < 32; c += 8)
      if (c < ncol) store_half8(row + c, v + c);
    if (cb > lb) {
#pragma unroll
      for (int c = 0; c < 32; ++c)
        if (c < ncol) h[(int64_t)(col0 + c) * g.ld + lane] = to_half(v[c]);
    }
    return;
  }
  const bool in = lane < g.lanes;
  const int safe = min(lane, g.lanes - 1);      // loads of lanes past the edge read a neighbour's values and drop them
  const int me = threadIdx.x & 31;
  if (kEpi == EPI_CODED) {
    const float sl = g.scale_lane ? g.scale_lane[safe] : 1.f;
    const float sc = g.scale_col[col0 + min(me, ncol - 1)];
    const int64_t at = (int64_t)lane * g.out_lane + (int64_t)col0 * g.out_col;
#pragma unroll
    for (int c = 0; c < 32; ++c) {
      const float v = (float)(int)acc[c] * __shfl_sync(0xFFFFFFFFu, sc, c) * sl;
      if (!in || c >= ncol) continue;
      if (g.out_bf16) ((__nv_bfloat16*)g.out)[at + c * g.out_col] = __float2bfloat16_rn(v);
      else ((float*)g.out)[at + c * g.out_col] = v;
    }
    return;
  }
  // X' = diag X + offdiag X: the product carries only the part off the diagonal, times kAScale * kXScale
  const float dc = g.d_in[z * g.d_stride + col0 + min(me, ncol - 1)];
  __half* lo = g.lo + z * g.stride + lane;
  float v[32];
  {
    __half oc[32], lc[32];
    load_column(g.o + z * g.stride + safe, col0, ncol, g.ld, oc);
    load_column(g.lo + z * g.stride + safe, col0, ncol, g.ld, lc);
#pragma unroll
    for (int c = 0; c < 32; ++c) {
      const float x = __half2float(oc[c]) + __half2float(lc[c]) * (1.f / kLoScale);
      v[c] = __shfl_sync(0xFFFFFFFFu, dc, c) * x + __uint_as_float(acc[c]) * (1.f / kAScale);
    }
  }
  if (kEpi == EPI_APPLY) {
    __half* h = g.h + z * g.stride + lane;
#pragma unroll
    for (int c = 0; c < 32; ++c) {
      if (in && c < ncol) {
        const int64_t i = (int64_t)(col0 + c) * g.ld;
        const __half hi = to_half(v[c]);
        h[i] = hi;
        lo[i] = to_half((v[c] - __half2float(hi)) * kLoScale);
      }
      v[c] = in ? v[c] * v[c] : 0.f;
    }
    // sums over the warp's 32 lanes, column c's in thread c
#pragma unroll
    for (int n = 16; n; n >>= 1)
#pragma unroll
      for (int i = 0; i < n; ++i) {
        const bool upper = me & n;
        const float give = upper ? v[i] : v[i + n], keep = upper ? v[i + n] : v[i];
        v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, n);
      }
    const int slot = (lane - me) / 32;
    if (me < ncol && slot < g.slots) g.row_sums[((int64_t)z * g.slots + slot) * g.d_stride + col0 + me] = v[0];
    return;
  }
  if (!in) return;
  const int64_t at = z * g.out_batch + (int64_t)lane * g.out_lane + (int64_t)col0 * g.out_col;
  if (kEpi == EPI_UPDATE) {
    float w[32];
#pragma unroll
    for (int c = 0; c < 32; ++c) w[c] = c < ncol ? ((const float*)g.out)[at + c * g.out_col] : 0.f;
#pragma unroll
    for (int c = 0; c < 32; ++c)
      if (c < ncol) ((float*)g.out)[at + c * g.out_col] = g.keep * w[c] - g.rate * (v[c] * (1.f / kXScale));
    return;
  }
#pragma unroll
  for (int c = 0; c < 32; ++c)
    if (c < ncol) {
      if (g.out_bf16) ((__nv_bfloat16*)g.out)[at + c * g.out_col] = __float2bfloat16_rn(v[c] * (1.f / kXScale));
      else ((float*)g.out)[at + c * g.out_col] = v[c] * (1.f / kXScale);
    }
}

template <int kCols>
__host__ __device__ constexpr int gemm_stages() { return (kSmemLimit - kSmemMisc) / ((kLanes + kCols) * kDepthBytes) > 8 ? 8 : (kSmemLimit - kSmemMisc) / ((kLanes + kCols) * kDepthBytes); }
template <int kCols>
__host__ __device__ constexpr int gemm_smem() { return gemm_stages<kCols>() * (kLanes + kCols) * kDepthBytes + kSmemMisc; }

template <int kCols, int kEpi>
__global__ void __launch_bounds__(kGemmThreads, 1)
k_gemm(const __grid_constant__ CUtensorMap map_p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ Gemm g) {
  constexpr bool kInt8 = kEpi == EPI_CODED;
  constexpr bool kMnMajor = kEpi == EPI_APPLY || kEpi == EPI_OUT || kEpi == EPI_UPDATE;   // P is stored with its lanes contiguous
  constexpr int kStages = gemm_stages<kCols>();
  constexpr int kPBytes = kLanes * kDepthBytes, kQBytes = kCols * kDepthBytes;
  constexpr int kDepth = kInt8 ? kDepthBytes : kDepthBytes / 2;      // elements of the contraction index per stage
  constexpr uint32_t kTmemCols = 2 * kCols < 32 ? 32 : 2 * kCols;

  extern __shared__ char smem_raw[];
  const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
  const uint32_t bars = base + kStages * (kPBytes + kQBytes);
  const uint32_t full = bars, empty = bars + 8 * kStages, tm_full = bars + 16 * kStages, tm_empty = tm_full + 16, drain = tm_empty + 16;
  char* gen = smem_raw + (base - smem_addr(smem_raw)) + kStages * (kPBytes + kQBytes);
  volatile uint32_t* words = (volatile uint32_t*)(gen + 16 * kStages + 48);      // [0] tensor-memory address, [1] give-up word
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const GiveUp give{words + 1, g.error};

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { bar_init(full + 8 * s, 1); bar_init(empty + 8 * s, 1); }
    for (int b = 0; b < 2; ++b) { bar_init(tm_full + 8 * b, 1); bar_init(tm_empty + 8 * b, kEpiWarps); }
    bar_init(drain, 1);
    words[1] = 0u;
    bar_init_fence();
    tma_prefetch(&map_p);
    tma_prefetch(&map_q);
  }
  if (warp == 1) tmem_alloc(smem_addr((const void*)words), kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = words[0];
  launch_wait();
  launch_next();

  const int total = g.tiles * g.batch;
  const int blocks_k = (g.depth + kDepth - 1) / kDepth;
  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (int t = blockIdx.x; t < total && ok; t += gridDim.x) {
        const Tile q = tile_at<kCols>(g, t);
        for (int kb = 0; kb < blocks_k; ++kb, ++it) {
          const uint32_t s = it % kStages;
          if (it >= (uint32_t)kStages && !(ok = bar_wait(empty + 8 * s, (it / kStages - 1) & 1, give))) break;
          const uint32_t dst = base + s * (kPBytes + kQBytes), bar = full + 8 * s;
          bar_expect(bar, kPBytes + kQBytes);
          if (kMnMajor) {
            tma_load(dst, &map_p, q.l * kLanes, kb * kDepth, q.z, bar);
            tma_load(dst + kPBytes / 2, &map_p, q.l * kLanes + 64, kb * kDepth, q.z, bar);
          } else {
            tma_load(dst, &map_p, kb * kDepth, q.l * kLanes, q.z, bar);
          }
          tma_load(dst + kPBytes, &map_q, kb * kDepth, q.c * kCols, q.z, bar);
        }
      }
      if (!ok)
        for (uint32_t k = it > (uint32_t)kStages ? it - kStages : 0; k < it; ++k) bar_drain(full + 8 * (k % kStages), (k / kStages) & 1);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      constexpr uint32_t kDesc = instr_desc(kInt8, kMnMajor, kCols);
      uint32_t it = 0, n = 0;
      bool ok = true;
      for (int t = blockIdx.x; t < total && ok; t += gridDim.x, ++n) {
        const uint32_t b = n & 1;
        if (n >= 2 && !(ok = bar_wait(tm_empty + 8 * b, (n / 2 - 1) & 1, give))) break;
        tc_fence_after();
        for (int kb = 0; kb < blocks_k; ++kb, ++it) {
          const uint32_t s = it % kStages;
          if (!(ok = bar_wait(full + 8 * s, (it / kStages) & 1, give))) break;
          tc_fence_after();
          const uint32_t src = base + s * (kPBytes + kQBytes);
          // one instruction takes 32 bytes of the contraction index: 16 steps of an MN-major tile are 2048 bytes on
          const uint64_t dp = smem_desc(src, kMnMajor ? kPBytes / 2 : 16), dq = smem_desc(src + kPBytes, 16);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            tc_mma<kInt8>(tmem + b * kCols, dp + (kMnMajor ? k * (2048 >> 4) : k * 2), dq + k * 2, kDesc, kb || k);
          tc_commit(empty + 8 * s);
        }
        if (ok) tc_commit(tm_full + 8 * b);
      }
      if (!ok) {
        tc_commit(drain);
        bar_drain(drain, 0);
      }
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3;       // the lanes of tensor memory that this warp may read
    const int first = (warp - 2) / 4 * 32;
    uint32_t n = 0;
    for (int t = blockIdx.x; t < total; t += gridDim.x, ++n) {
      const uint32_t b = n & 1;
      const Tile q = tile_at<kCols>(g, t);
      const int row = q.l * kLanes + quarter * 32 + lane;
      float diag = 0.f;
      if (kEpi == EPI_GRAM && q.l == q.c * kCols / kLanes) diag = gram_diagonal(g, q.z, row);
      if (kEpi == EPI_GRAM && kCols > kLanes && q.l == q.c * kCols / kLanes + 1) diag = gram_diagonal(g, q.z, row);
      if (!__all_sync(0xFFFFFFFFu, bar_wait(tm_full + 8 * b, (n / 2) & 1, give))) break;
      tc_fence_after();
#pragma unroll 1
      for (int c = first; c < kCols; c += 32 * (kEpiWarps / 4)) {
        if (q.c * kCols + c >= g.cols) break;
        uint32_t acc[32];
        tmem_load32(tmem + b * kCols + c + ((uint32_t)(quarter * 32) << 16), acc);
        epilogue<kEpi>(g, q.z, row, q.c * kCols + c, diag, acc);
        __syncwarp();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive(tm_empty + 8 * b);
    }
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_free(tmem, kTmemCols);
}

}  // namespace mat
}  // namespace rtopk
