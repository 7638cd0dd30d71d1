// The tensor-core product of the matrix operators: D[lane][col] = sum_k P[lane][k] Q[col][k], 16-bit floating point
// with 32-bit sums or 8-bit integers with 32-bit integer sums, and what is done with D before it leaves the SM.
//
// One persistent block per SM, ten warps: one thread feeds a ring of shared-memory stages by TMA, one thread issues
// the products, eight warps turn finished tiles into results while the next tile is being multiplied (the accumulators
// lie twice in tensor memory).  D is always laid out so that the 32 lanes of a warp are neighbours in the result's rows:
// the stores are coalesced without a pass through shared memory.
//
// The mainloop is bound by what L2 gives the SMs (about 15 TB/s over all of them), not by the tensor cores: a block of 128 x 256
// reads 48 KB for 512 cycles' worth of 16-bit products.  So large products run in pairs of blocks (two SMs, one 256 x kCols tile):
// each block loads its own 128 rows of P and half of Q's rows, and the pair's first block issues the products for both.
//
// Small products leave SMs idle with one tile per block; there the contraction is cut into g.split parts, each block leaves its
// partial sums in scratch, and the block that comes last to a tile adds the parts in their order and goes on as usual.
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
  int split;                 // parts of the contraction, 1: whole
  uint32_t* parts;           // split: partial sums, [unit][col][lane]
  uint32_t* arrived;         // split: blocks that have left their part, per tile and block of a pair; zero between launches
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

// Of a triangular product: column tile c reaches the lane tiles 0 .. this - 1.
template <int kCols, int kTileLanes>
__host__ __device__ constexpr int tri_lane_tiles(int tiles_l, int c) {
  return ((c + 1) * kCols - 1) / kTileLanes + 1 < tiles_l ? ((c + 1) * kCols - 1) / kTileLanes + 1 : tiles_l;
}

struct Tile { int l, c, z, part; };

// lanes: of a tile, 128 or 256
template <int kCols, int kTileLanes>
__device__ __forceinline__ Tile tile_at(const Gemm& g, int unit) {
  Tile r;
  const int t = unit / g.split;
  r.part = unit - t * g.split;
  r.z = t / g.tiles;
  int k = t - r.z * g.tiles;
  if (!g.tri) {
    r.c = k / g.tiles_l;
    r.l = k - r.c * g.tiles_l;
    return r;
  }
  for (r.c = 0;; ++r.c) {
    const int n = tri_lane_tiles<kCols, kTileLanes>(g.tiles_l, r.c);
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
  bool in = lane < g.lanes;
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
  int n = ncol;
  int64_t at = z * g.out_batch + (int64_t)lane * g.out_lane + (int64_t)col0 * g.out_col, step = g.out_col;
  if (g.out_lane != 1) {      // the result's rows run along the columns: turn the 32 x 32 block round
    in = me < ncol;
    n = min(32, g.lanes - (lane - me));
    at = z * g.out_batch + (int64_t)(lane - me) * g.out_lane + (int64_t)(col0 + me) * g.out_col, step = g.out_lane;
#pragma unroll
    for (int k = 16; k; k >>= 1)
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (!(i & k)) {
          const bool upper = me & k;
          const float got = __shfl_xor_sync(0xFFFFFFFFu, upper ? v[i] : v[i | k], k);
          if (upper) v[i] = got;
          else v[i | k] = got;
        }
  }
  if (!in) return;
  if (kEpi == EPI_UPDATE) {
    float w[32];
#pragma unroll
    for (int c = 0; c < 32; ++c) w[c] = ((const float*)g.out)[at + min(c, n - 1) * step];
#pragma unroll
    for (int c = 0; c < 32; ++c)
      if (c < n) ((float*)g.out)[at + c * step] = g.keep * w[c] - g.rate * (v[c] * (1.f / kXScale));
    return;
  }
#pragma unroll
  for (int c = 0; c < 32; ++c)
    if (c < n) {
      if (g.out_bf16) ((__nv_bfloat16*)g.out)[at + c * step] = __float2bfloat16_rn(v[c] * (1.f / kXScale));
      else ((float*)g.out)[at + c * step] = v[c] * (1.f / kXScale);
    }
}

template <int kCols, bool kPair>
struct GemmShape {
  static constexpr int kTileLanes = kPair ? 2 * kLanes : kLanes;
  static constexpr int kQRows = kPair ? kCols / 2 : kCols;             // rows of Q in one block's stage
  static constexpr int kPBytes = kLanes * kDepthBytes, kQBytes = kQRows * kDepthBytes, kStageBytes = kPBytes + kQBytes;
  static constexpr int kFit = (kSmemLimit - kSmemMisc) / kStageBytes;
  static constexpr int kStages = kFit > 8 ? 8 : kFit;
  static constexpr int kSmem = kStages * kStageBytes + kSmemMisc;
};

template <int kCols, bool kPair, int kEpi>
__global__ void __launch_bounds__(kGemmThreads, 1)
k_gemm(const __grid_constant__ CUtensorMap map_p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ Gemm g) {
  using S = GemmShape<kCols, kPair>;
  constexpr bool kInt8 = kEpi == EPI_CODED;
  constexpr bool kMnMajor = kEpi == EPI_APPLY || kEpi == EPI_OUT || kEpi == EPI_UPDATE;   // P is stored with its lanes contiguous
  constexpr int kStages = S::kStages;
  constexpr int kDepth = kInt8 ? kDepthBytes : kDepthBytes / 2;      // elements of the contraction index per stage
  constexpr int kBlocks = kPair ? 2 : 1;
  constexpr uint32_t kTmemCols = 2 * kCols;

  extern __shared__ char smem_raw[];
  const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
  const uint32_t full = base + kStages * S::kStageBytes, empty = full + 8 * kStages, tm_full = empty + 8 * kStages, tm_empty = tm_full + 16, drain = tm_empty + 16, meet = drain + 8;
  char* gen = smem_raw + (base - smem_addr(smem_raw)) + kStages * S::kStageBytes;
  // [0] tensor-memory address, [1] give-up word, [2] whether this block came last to a split tile
  volatile uint32_t* words = (volatile uint32_t*)(gen + 16 * kStages + 64);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = kPair ? rank_in_pair() : 0;
  const GiveUp give{words + 1, g.error};

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { bar_init(full + 8 * s, 1); bar_init(empty + 8 * s, 1); }
    for (int b = 0; b < 2; ++b) { bar_init(tm_full + 8 * b, 1); bar_init(tm_empty + 8 * b, kBlocks * kEpiWarps); }
    bar_init(drain, 1);
    bar_init(meet, kEpiWarps);
    words[1] = 0u;
    bar_init_fence();
    tma_prefetch(&map_p);
    tma_prefetch(&map_q);
  }
  if (warp == 1) tmem_alloc<kPair>(smem_addr((const void*)words), kTmemCols);
  tc_fence_before();
  if (kPair) pair_sync();
  else __syncthreads();
  tc_fence_after();
  const uint32_t tmem = words[0];
  launch_wait();
  launch_next();

  const int total = g.tiles * g.batch * g.split;
  const int first = blockIdx.x / kBlocks, step = gridDim.x / kBlocks;
  const int all_k = (g.depth + kDepth - 1) / kDepth, part_k = (all_k + g.split - 1) / g.split;
  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (int u = first; u < total && ok; u += step) {
        const Tile q = tile_at<kCols, S::kTileLanes>(g, u);
        const int k1 = min(all_k, (q.part + 1) * part_k);
        const int p_row = q.l * S::kTileLanes + rank * kLanes, q_row = q.c * kCols + rank * S::kQRows;
        for (int kb = q.part * part_k; kb < k1; ++kb, ++it) {
          const uint32_t s = it % kStages;
          if (it >= (uint32_t)kStages && !(ok = bar_wait(empty + 8 * s, (it / kStages - 1) & 1, give))) break;
          const uint32_t dst = base + s * S::kStageBytes;
          if (rank == 0) bar_expect(full + 8 * s, kBlocks * S::kStageBytes);
          const uint32_t bar = kPair ? first_of_pair(full + 8 * s) : full + 8 * s;
          if (kMnMajor) {
            tma_load<kPair>(dst, &map_p, p_row, kb * kDepth, q.z, bar);
            tma_load<kPair>(dst + S::kPBytes / 2, &map_p, p_row + 64, kb * kDepth, q.z, bar);
          } else {
            tma_load<kPair>(dst, &map_p, kb * kDepth, p_row, q.z, bar);
          }
          tma_load<kPair>(dst + S::kPBytes, &map_q, kb * kDepth, q_row, q.z, bar);
        }
      }
      if (!ok) {
        if (rank == 0) {
          for (uint32_t k = it > (uint32_t)kStages ? it - kStages : 0; k < it; ++k) bar_drain(full + 8 * (k % kStages), (k / kStages) & 1);
        } else {      // this block's copies report to the other one: give them time
          const uint64_t t0 = now_ns();
          while (now_ns() - t0 < 1000000ull) {}
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      constexpr uint32_t kDesc = instr_desc(kInt8, kMnMajor, S::kTileLanes, kCols);
      uint32_t it = 0, n = 0;
      bool ok = true;
      for (int u = first; u < total && ok; u += step, ++n) {
        const Tile q = tile_at<kCols, S::kTileLanes>(g, u);
        const int k0 = q.part * part_k, k1 = min(all_k, k0 + part_k);
        const uint32_t b = n & 1;
        if (n >= 2 && !(ok = bar_wait(tm_empty + 8 * b, (n / 2 - 1) & 1, give))) break;
        tc_fence_after();
        for (int kb = k0; kb < k1; ++kb, ++it) {
          const uint32_t s = it % kStages;
          if (!(ok = bar_wait(full + 8 * s, (it / kStages) & 1, give))) break;
          tc_fence_after();
          const uint32_t src = base + s * S::kStageBytes;
          // one instruction takes 32 bytes of the contraction index: 16 steps of an MN-major tile are 2048 bytes on
          const uint64_t dp = smem_desc(src, kMnMajor ? S::kPBytes / 2 : 16), dq = smem_desc(src + S::kPBytes, 16);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            tc_mma<kPair, kInt8>(tmem + b * kCols, dp + (kMnMajor ? k * (2048 >> 4) : k * 2), dq + k * 2, kDesc, kb > k0 || k);
          tc_commit<kPair>(empty + 8 * s);
        }
        if (ok) tc_commit<kPair>(tm_full + 8 * b);
      }
      if (!ok) {
        tc_commit<kPair>(drain);
        bar_drain(drain, 0);
      }
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3;       // the lanes of tensor memory that this warp may read
    const int chunk0 = (warp - 2) / 4 * 32;
    uint32_t n = 0, met = 0;
    // all epilogue warps, with the limit of every wait
    auto together = [&]() {
      __syncwarp();
      if (lane == 0) bar_arrive(meet);
      return __all_sync(0xFFFFFFFFu, bar_wait(meet, met++ & 1, give)) != 0;
    };
    for (int u = first; u < total; u += step, ++n) {
      const uint32_t b = n & 1;
      const Tile q = tile_at<kCols, S::kTileLanes>(g, u);
      const int in_tile = quarter * 32 + lane;
      const int row0 = q.l * S::kTileLanes + rank * kLanes, row = row0 + in_tile;
      float diag = 0.f;
      if (kEpi == EPI_GRAM && q.c * kCols < row0 + kLanes && row0 < (q.c + 1) * kCols) diag = gram_diagonal(g, q.z, row);
      if (!__all_sync(0xFFFFFFFFu, bar_wait(tm_full + 8 * b, (n / 2) & 1, give))) break;
      tc_fence_after();
      const uint32_t from = tmem + b * kCols + ((uint32_t)(quarter * 32) << 16);
      const int cols = min(kCols, g.cols - q.c * kCols);
      if (g.split == 1) {
#pragma unroll 1
        for (int c = chunk0; c < cols; c += 32 * (kEpiWarps / 4)) {
          uint32_t acc[32];
          tmem_load32(from + c, acc);
          epilogue<kEpi>(g, q.z, row, q.c * kCols + c, diag, acc);
          __syncwarp();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (kPair) bar_arrive_cluster(first_of_pair(tm_empty + 8 * b));
          else bar_arrive(tm_empty + 8 * b);
        }
        continue;
      }
      const int64_t part_words = (int64_t)kCols * S::kTileLanes;
      uint32_t* mine = g.parts + u * part_words + rank * kLanes + in_tile;
#pragma unroll 1
      for (int c = chunk0; c < cols; c += 32 * (kEpiWarps / 4)) {
        uint32_t acc[32];
        tmem_load32(from + c, acc);
#pragma unroll
        for (int i = 0; i < 32; ++i) mine[(c + i) * S::kTileLanes] = acc[i];
      }
      tc_fence_before();
      __threadfence();
      if (!together()) break;
      if (warp == 2 && lane == 0) {
        uint32_t* seen = g.arrived + (u / g.split) * kBlocks + rank;
        const uint32_t before = atomicAdd(seen, 1u);
        if (before + 1 == (uint32_t)g.split) *seen = 0u;
        words[2] = before + 1 == (uint32_t)g.split;
      }
      if (!together()) break;
      const bool last = words[2] != 0u;
      if (lane == 0) {
        if (kPair) bar_arrive_cluster(first_of_pair(tm_empty + 8 * b));
        else bar_arrive(tm_empty + 8 * b);
      }
      if (!together()) break;      // words[2] may change from here on
      if (!last) continue;
      __threadfence();
      const uint32_t* parts = g.parts + (u - q.part) * part_words + rank * kLanes + in_tile;
#pragma unroll 1
      for (int c = chunk0; c < cols; c += 32 * (kEpiWarps / 4)) {
        uint32_t acc[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[i] = __ldcg(parts + (c + i) * S::kTileLanes);
        for (int k = 1; k < g.split; ++k) {
          const uint32_t* next = parts + k * part_words;
          uint32_t w[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) w[i] = __ldcg(next + (c + i) * S::kTileLanes);
#pragma unroll
          for (int i = 0; i < 32; ++i)
            acc[i] = kInt8 ? acc[i] + w[i] : __float_as_uint(__uint_as_float(acc[i]) + __uint_as_float(w[i]));
        }
        epilogue<kEpi>(g, q.z, row, q.c * kCols + c, diag, acc);
        __syncwarp();
      }
    }
    __syncwarp();
  }
  tc_fence_before();
  if (kPair) pair_sync();
  else __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_free<kPair>(tmem, kTmemCols);
}

}  // namespace mat
}  // namespace rtopk
