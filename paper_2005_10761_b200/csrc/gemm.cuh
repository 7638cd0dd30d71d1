// The tensor-core product of the matrix operators: D[lane][col] = sum_k P[lane][k] Q[col][k], 16-bit floating point
// with 32-bit sums or 8-bit integers with 32-bit integer sums, and what is done with D before it leaves the SM.
//
// One persistent block per SM, ten warps: one feeds a ring of shared-memory stages by TMA, one issues the products, eight
// turn finished tiles into results while the next tile is being multiplied (the accumulators lie twice in tensor memory).  D
// is always laid out so that the 32 lanes of a warp are neighbours in the result's rows: the stores are coalesced without a
// pass through shared memory.
//
// An SM gets 64 bytes a cycle from L2 (a step of 128 bytes of the contraction index: 0.19 us for the 24 KB of a 128-column
// stage), so a block of 128 x 256 alone would wait for its 48 KB half of the time.  Large products run in pairs of blocks (two SMs,
// one 256 x kCols tile): each block loads its own 128 rows of P and half of Q's rows, and the pair's first block issues the
// products for both; 256 columns then take 0.27 to 0.30 us a step, the tensor cores' 512 cycles.  Both figures need the loops of
// the feeding and the issuing warp to keep their addresses in uniform registers; run by one thread they took 0.31 and 0.41 us.
//
// What bounds it: large products the tensor cores, and under load the card's power (codes 8192 x 4096 by 4096 x 8192 0.19 ms, 2.9
// Pop/s, where a short burst does 3.6); products of one or two waves the boundary between launches (1.4 us), the first bytes
// (0.6 us), the results behind the last products (256 columns of X 6 to 8 us: 10 bytes an entry, from and to L2, all SMs at once)
// and tiles that do not fill the SMs.  In the smallest, fetching instructions for the first time counts: one copy of the results'
// code for whole and split tiles, and waiting for the launch before only where a role first has to, took 256 x 256 from 84 to 70 us (66 now).
//
// Small products leave SMs idle with one tile per block; there the contraction is cut into g.split parts, each block leaves its
// partial sums in scratch, and the block that comes last to a tile adds the parts in their order and goes on as usual (Gram
// product of 1500 x 10000: 59 us whole, 39 us in three parts).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "tensorcore.cuh"

namespace rtopk {
namespace mat {

constexpr int kEpiWarps = 8;                // two for each quarter of the accumulator's lanes, taking its column chunks in turn
constexpr int kGemmThreads = 64 + 32 * kEpiWarps;
constexpr int kLanes = 128;                 // rows of an accumulator tile (tensor-memory lanes)
constexpr int kDepthBytes = 128;            // bytes of the contraction index per stage and row: one swizzle row
constexpr int kSmemLimit = 227 * 1024;
constexpr int kSmemMisc = 1024 + 2048;      // alignment slack, barriers, the epilogue's columns

// Scales that keep 16-bit entries away from the subnormal range: X is held times 32 and its Gram matrix and the
// polynomial of it times 1024.  ||X||_F = 1 at the start, so an entry of a 10000 x 1500 X is about 2.6e-4; afterwards
// singular values stay below about 1.3, so nothing comes near the largest 16-bit number.
constexpr float kXScale = 32.f, kAScale = 1024.f;

enum Epi : int {
  EPI_GRAM = 0,    // A = X X^T: entries off the diagonal in 16 bits, the diagonal (from the unrounded X) in 32
  EPI_POLY = 1,    // a + b A + c A^2, in the same form
  EPI_APPLY = 2,   // X <- (that) X, in 32 bits and in 16
  EPI_OUT = 3,     // the last X, into the caller's matrix
  EPI_UPDATE = 4,  // the last X, into the caller's weights
  EPI_CODED = 5    // 8-bit codes: times the two scales
};

struct Gemm {
  int lanes, cols, depth;    // D is lanes x cols; depth in elements
  int batch, tiles_l, tiles_c, tiles;   // tiles per batch entry
  int tri;                   // only tiles that reach the upper triangle (col >= lane)
  int p_early;               // P is not written by the kernel before this one: its first stages are loaded ahead of launch_wait()
  int free_start;            // nothing here touches what the kernel before this one reads or writes: launch_wait() comes last
  int split;                 // parts of the contraction, 1: whole
  uint32_t* parts;           // split: partial sums, [unit][col][lane]
  uint32_t* arrived;         // split: blocks that have left their part, per tile and block of a pair; zero between launches
  int test_giveup;           // tests only: the first wait for a stage counts as run out, and one block of each pair stops feeding early
  uint32_t* error;
  // epilogue operands
  const __half* o;           // POLY: A off the diagonal
  float* x;                  // APPLY / OUT / UPDATE: X in 32 bits (APPLY: replaced in place)
  __half* h;                 // 16-bit result
  int64_t ld, stride;        // of o, x, h
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
// tile's products are waited for.  32 at a time, their sums in binary64: in one chain of binary32 sums 2^19 equal ones came out 1 %
// off (a row of 2^24 ones), and 2^24 would be the most it reaches.
__device__ __forceinline__ float gram_diagonal(const Gemm& g, int z, int lane) {
  if (lane >= g.lanes) return 0.f;
  const float* sums = g.row_sums + (int64_t)z * g.slots * g.d_stride + lane;
  double d = 0.0;
  int i = 0;
  for (; i + 32 <= g.slots; i += 32) {
    float v[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = sums[(i + j) * g.d_stride];
#pragma unroll
    for (int k = 16; k; k >>= 1)
#pragma unroll
      for (int j = 0; j < k; ++j) v[j] += v[j + k];
    d += v[0];
  }
  for (; i < g.slots; ++i) d += sums[i * g.d_stride];
  return (float)d * (1.f / kAScale);
}

// 32 entries of one lane, `step` apart (past the edge the last one again): all loads are under way before the first is used.
template <bool kFull, class T>
__device__ __forceinline__ void load_strip(const T* p, int n, int64_t step, T (&v)[32]) {
#pragma unroll
  for (int c = 0; c < 32; ++c) {
    v[c] = *p;
    if (kFull || c + 1 < n) p += step;
  }
}
template <bool kFull, class T, class F>
__device__ __forceinline__ void store_strip(T* p, int n, int64_t step, F value) {
#pragma unroll
  for (int c = 0; c < 32; ++c) {
    if (kFull || c < n) *p = value(c);
    p += step;
  }
}

// What the results of 32 columns need beside the products.  Read ahead: for a tile's first columns while its products are
// still being formed, then for the next columns while the present ones are finished.
template <int kEpi>
struct Ahead {
  typename std::conditional<kEpi == EPI_POLY, __half, float>::type at[kEpi == EPI_POLY || kEpi == EPI_APPLY || kEpi == EPI_OUT || kEpi == EPI_UPDATE ? 32 : 1];
  float col;             // of column `threadIdx & 31`: its entry of the diagonal, or its scale
};

template <int kEpi, bool kFull>
__device__ __forceinline__ void read_ahead(const Gemm& g, int z, int lane, int col0, int n, Ahead<kEpi>& ahead) {
  const int me = threadIdx.x & 31;
  const int safe = kFull ? lane : min(lane, g.lanes - 1), my_col = col0 + (kFull ? me : min(me, n - 1));
  if constexpr (kEpi == EPI_POLY) {
    if (col0 / kLanes < lane / kLanes) return;
    load_strip<kFull>(g.o + z * g.stride + col0 * g.ld + safe, n, g.ld, ahead.at);
  } else if constexpr (kEpi == EPI_APPLY || kEpi == EPI_OUT || kEpi == EPI_UPDATE) {
    load_strip<kFull>((const float*)g.x + z * g.stride + col0 * g.ld + safe, n, g.ld, ahead.at);
  }
  if constexpr (kEpi == EPI_CODED) ahead.col = g.scale_col[my_col];
  else if constexpr (kEpi != EPI_GRAM) ahead.col = g.d_in[z * g.d_stride + my_col];
}

// 32 columns (col0 ..) of lane `lane` of one tile; all 32 threads of the warp come here, each with its lane.  kFull: the
// warp's lanes and columns all exist.  `n` of the columns do; loads of lanes that do not read a neighbour's values.
// `of_lane`: the lane's entry of the diagonal (GRAM: of the result's), or its scale.
template <int kEpi, bool kFull>
__device__ __forceinline__ void epilogue(const Gemm& g, int z, int lane, int col0, int n, float of_lane, float* cols, const Ahead<kEpi>& ahead, const uint32_t (&acc)[32]) {
  const int me = threadIdx.x & 31;
  bool in = kFull || lane < g.lanes;
  float of_col[kEpi == EPI_GRAM ? 1 : 32];      // every column's number in every thread: by way of the warp's place in shared memory
  if constexpr (kEpi != EPI_GRAM) {
    cols[me] = ahead.col;
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 32; c += 4) {
      const float4 q = *(const float4*)(cols + c);
      of_col[c] = q.x, of_col[c + 1] = q.y, of_col[c + 2] = q.z, of_col[c + 3] = q.w;
    }
  }
  float v[32];
  if constexpr (kEpi == EPI_GRAM || kEpi == EPI_POLY) {
    // Symmetric result: a 128-wide block of columns left of this lane's block is the mirror image of another tile.
    const int lb = lane / kLanes, cb = col0 / kLanes;
    if (cb < lb) return;
    if constexpr (kEpi == EPI_GRAM) {
#pragma unroll
      for (int c = 0; c < 32; ++c) v[c] = __uint_as_float(acc[c]);
    } else {
      const float dl = g.b + g.c * of_lane, scale = g.c * (1.f / kAScale);
#pragma unroll
      for (int c = 0; c < 32; ++c) v[c] = scale * __uint_as_float(acc[c]) + fmaf(g.c, of_col[c], dl) * __half2float(ahead.at[c]);
    }
    if (cb == lb && in && lane >= col0 && lane < col0 + n) {
      float q = 0.f;
#pragma unroll
      for (int c = 0; c < 32; ++c)
        if (lane == col0 + c) {
          q = __uint_as_float(acc[c]) * (1.f / kAScale);
          v[c] = 0.f;
        }
      g.d_out[z * g.d_stride + lane] = kEpi == EPI_GRAM ? of_lane : g.a + g.b * of_lane + g.c * (of_lane * of_lane + q * (1.f / kAScale));
    }
    if (!in) return;
    // row `lane`, columns col0 ..: the row stride is a multiple of 8, so the padding takes whole vectors
    __half* row = g.h + z * g.stride + lane * g.ld + col0;
#pragma unroll
    for (int c = 0; c < 32; c += 8)
      if (kFull || c < n) store_half8(row + c, v + c);
    if (cb > lb) store_strip<kFull>(g.h + z * g.stride + col0 * g.ld + lane, n, g.ld, [&](int c) { return to_half(v[c]); });
  } else if constexpr (kEpi == EPI_CODED) {
#pragma unroll
    for (int c = 0; c < 32; ++c) v[c] = (float)(int)acc[c] * of_col[c] * of_lane;
    if (!in) return;
    const int64_t at = lane + col0 * g.out_col;
    if (g.out_bf16) store_strip<kFull>((__nv_bfloat16*)g.out + at, n, g.out_col, [&](int c) { return __float2bfloat16_rn(v[c]); });
    else store_strip<kFull>((float*)g.out + at, n, g.out_col, [&](int c) { return v[c]; });
  } else {
    // X' = diag X + offdiag X: the product carries only the part off the diagonal, times kAScale * kXScale.  X of the diagonal's
    // term is the one in 32 bits, in the last product too: read there from its 16-bit form, a matrix with orthogonal rows would come
    // out 2.1e-4 off instead of 1e-6 (and 1500 x 10000 would take 583 instead of 601 us).
#pragma unroll
    for (int c = 0; c < 32; ++c) v[c] = of_col[c] * ahead.at[c] + __uint_as_float(acc[c]) * (1.f / kAScale);
    if constexpr (kEpi == EPI_APPLY) {
      if (in) {
        store_strip<kFull>(g.x + z * g.stride + col0 * g.ld + lane, n, g.ld, [&](int c) { return v[c]; });
        store_strip<kFull>(g.h + z * g.stride + col0 * g.ld + lane, n, g.ld, [&](int c) { return to_half(v[c]); });
      }
#pragma unroll
      for (int c = 0; c < 32; ++c) v[c] = in ? v[c] * v[c] : 0.f;
      // sums over the warp's 32 lanes, column c's in thread c
#pragma unroll
      for (int k = 16; k; k >>= 1)
#pragma unroll
        for (int i = 0; i < k; ++i) {
          const bool upper = me & k;
          const float give = upper ? v[i] : v[i + k], keep = upper ? v[i + k] : v[i];
          v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, k);
        }
      const int slot = (lane - me) / 32;
      if (kFull || (me < n && slot < g.slots)) g.row_sums[((int64_t)z * g.slots + slot) * g.d_stride + col0 + me] = v[0];
    } else {
      int64_t at = z * g.out_batch + lane * g.out_lane + col0 * g.out_col, step = g.out_col;
      if (g.out_lane != 1) {      // the result's rows run along the columns: turn the 32 x 32 block round
        in = kFull || me < n;
        n = kFull ? 32 : min(32, g.lanes - (lane - me));
        at = z * g.out_batch + (lane - me) * g.out_lane + (col0 + me) * g.out_col, step = g.out_lane;
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
      if (!in || n <= 0) return;
      if constexpr (kEpi == EPI_UPDATE) {
        float w[32];
        load_strip<kFull>((const float*)g.out + at, n, step, w);
        const float rate = g.rate * (1.f / kXScale);
        store_strip<kFull>((float*)g.out + at, n, step, [&](int c) { return g.keep * w[c] - rate * v[c]; });
      } else if (g.out_bf16) {
        store_strip<kFull>((__nv_bfloat16*)g.out + at, n, step, [&](int c) { return __float2bfloat16_rn(v[c] * (1.f / kXScale)); });
      } else {
        store_strip<kFull>((float*)g.out + at, n, step, [&](int c) { return v[c] * (1.f / kXScale); });
      }
    }
  }
}

template <int kCols, bool kPair>
struct GemmShape {
  static constexpr int kTileLanes = kPair ? 2 * kLanes : kLanes;
  static constexpr int kQRows = kPair ? kCols / 2 : kCols;             // rows of Q in one block's stage
  static constexpr int kPBytes = kLanes * kDepthBytes, kQBytes = kQRows * kDepthBytes, kStageBytes = kPBytes + kQBytes;
  static constexpr int kFit = (kSmemLimit - kSmemMisc) / kStageBytes;
  static constexpr int kStages = kFit > 8 ? 8 : kFit;
  static constexpr int kSmem = kStages * kStageBytes + 2048;      // the rest is static
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
  __shared__ __align__(16) float epi_cols[kEpiWarps][32];
  const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
  const uint32_t full = base + kStages * S::kStageBytes, empty = full + 8 * kStages, tm_full = empty + 8 * kStages, tm_empty = tm_full + 16, drain = tm_empty + 16, meet = drain + 8;
  char* gen = smem_raw + (base - smem_addr(smem_raw)) + kStages * S::kStageBytes;
  // [0] tensor-memory address, [1] give-up word, [2] whether this block came last to a split tile, [3] stages it has asked for
  volatile uint32_t* words = (volatile uint32_t*)(gen + 16 * kStages + 64);
  const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;      // the same for all of a warp, and known to be
  const uint32_t rank = kPair ? rank_in_cluster() : 0;
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
  if (kPair) cluster_sync();
  else __syncthreads();
  tc_fence_after();
  const uint32_t tmem = words[0];

  const int total = g.tiles * g.batch * g.split;
  const int first = blockIdx.x / kBlocks, step = gridDim.x / kBlocks;
  const int all_k = (g.depth + kDepth - 1) / kDepth, part_k = (all_k + g.split - 1) / g.split;
  auto load_p = [&](uint32_t s, const Tile& q, int kb) {
    const uint32_t dst = base + s * S::kStageBytes, bar = kPair ? first_of_pair(full + 8 * s) : full + 8 * s;
    const int row = q.l * S::kTileLanes + rank * kLanes;
    if (rank == 0) bar_expect(full + 8 * s, kBlocks * S::kStageBytes);
    if (kMnMajor) {
      tma_load<kPair>(dst, &map_p, row, kb * kDepth, q.z, bar);
      tma_load<kPair>(dst + S::kPBytes / 2, &map_p, row + 64, kb * kDepth, q.z, bar);
    } else {
      tma_load<kPair>(dst, &map_p, kb * kDepth, row, q.z, bar);
    }
  };
  uint32_t early = 0;      // stages whose P is under way
  if (g.p_early && warp == 0 && first < total) {
    const Tile q = tile_at<kCols, S::kTileLanes>(g, first);
    const int k0 = q.part * part_k, n = min(kStages, min(all_k, k0 + part_k) - k0);
    for (; early < (uint32_t)n; ++early)
      if (elect_one()) load_p(early, q, k0 + early);
  }
  // Each role waits for the kernel before this one only where it first needs to: what leads there, and the instructions it
  // takes, are behind it by then.
  auto follow = [&]() {
    launch_wait();
    launch_next();
  };
  if (warp == 0) {
    uint32_t it = 0;
    const uint32_t feed = kPair && g.test_giveup && ((first ^ rank) & 1) ? max(1u, early) : ~0u;
    bool ok = true;
    for (int u = first; u < total && ok; u += step) {
      const Tile q = tile_at<kCols, S::kTileLanes>(g, u);
      const int k1 = min(all_k, (q.part + 1) * part_k);
      if (it == 0 && !g.free_start) follow();
#pragma unroll 1
      for (int kb = q.part * part_k; kb < k1; ++kb, ++it) {
        const uint32_t s = it % kStages;
        if (it >= (uint32_t)kStages && !(ok = __all_sync(0xFFFFFFFFu, bar_wait(empty + 8 * s, (it / kStages - 1) & 1, give)))) break;
        if (!(ok = it < feed)) break;
        if (elect_one()) {
          if (it >= early) load_p(s, q, kb);
          tma_load<kPair>(base + s * S::kStageBytes + S::kPBytes, &map_q, kb * kDepth, q.c * kCols + rank * S::kQRows, q.z, kPair ? first_of_pair(full + 8 * s) : full + 8 * s);
        }
        __syncwarp();
      }
    }
    if (lane == 0) words[3] = it;
    __syncwarp();
  } else if (warp == 1) {
    if (!g.free_start) follow();      // before the first wait with a limit, which is not to count what is left of that kernel
    if (rank == 0) {
      constexpr uint32_t kDesc = instr_desc(kInt8, kMnMajor, S::kTileLanes, kCols);
      uint32_t it = 0, n = 0;
      bool ok = !g.test_giveup || give_up(give);
      for (int u = first; u < total && ok; u += step, ++n) {
        const Tile q = tile_at<kCols, S::kTileLanes>(g, u);
        const int k0 = q.part * part_k, k1 = min(all_k, k0 + part_k);
        const uint32_t b = n & 1;
        if (n >= 2 && !(ok = __all_sync(0xFFFFFFFFu, bar_wait(tm_empty + 8 * b, (n / 2 - 1) & 1, give)))) break;
        tc_fence_after();
#pragma unroll 1
        for (int kb = k0; kb < k1; ++kb, ++it) {
          const uint32_t s = it % kStages;
          if (!(ok = __all_sync(0xFFFFFFFFu, bar_wait(full + 8 * s, (it / kStages) & 1, give)))) break;
          tc_fence_after();
          const uint32_t src = base + s * S::kStageBytes;
          // one instruction takes 32 bytes of the contraction index: 16 steps of an MN-major tile are 2048 bytes on
          const uint64_t dp = smem_desc(src, kMnMajor ? S::kPBytes / 2 : 16), dq = smem_desc(src + S::kPBytes, 16);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              tc_mma<kPair, kInt8>(tmem + b * kCols, dp + (kMnMajor ? k * (2048 >> 4) : k * 2), dq + k * 2, kDesc, kb > k0 || k);
            tc_commit<kPair>(empty + 8 * s);
          }
          __syncwarp();
        }
        if (ok && elect_one()) tc_commit<kPair>(tm_full + 8 * b);
        __syncwarp();
      }
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3;       // the lanes of tensor memory that this warp may read
    const int chunk0 = (warp - 2) / 4 * 32;
    float* cols_at = epi_cols[warp - 2];
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
      constexpr int kNext = 32 * (kEpiWarps / 4);
      const int cols = min(kCols, g.cols - q.c * kCols);
      const bool lanes_full = row0 + kLanes <= g.lanes;
      float of_lane = 1.f;
      if (n == 0 && !g.free_start) follow();
      if (kEpi == EPI_GRAM) {
        if (q.c * kCols < row0 + kLanes && row0 < (q.c + 1) * kCols) of_lane = gram_diagonal(g, q.z, row);
      } else if (kEpi == EPI_POLY) {
        of_lane = g.d_in[q.z * g.d_stride + min(row, g.lanes - 1)];
      } else if (kEpi == EPI_CODED) {
        if (g.scale_lane) of_lane = g.scale_lane[min(row, g.lanes - 1)];
      }
      auto read = [&](int c, Ahead<kEpi>& ahead) {
        if (c >= cols) return;
        if (lanes_full && c + 32 <= cols) read_ahead<kEpi, true>(g, q.z, row, q.c * kCols + c, 32, ahead);
        else read_ahead<kEpi, false>(g, q.z, row, q.c * kCols + c, min(32, cols - c), ahead);
      };
      auto finish = [&](int c, const Ahead<kEpi>& ahead, const uint32_t(&acc)[32]) {
        if (lanes_full && c + 32 <= cols) epilogue<kEpi, true>(g, q.z, row, q.c * kCols + c, 32, of_lane, cols_at, ahead, acc);
        else epilogue<kEpi, false>(g, q.z, row, q.c * kCols + c, min(32, cols - c), of_lane, cols_at, ahead, acc);
        __syncwarp();
      };
      Ahead<kEpi> ahead;
      read(chunk0, ahead);
      if (!__all_sync(0xFFFFFFFFu, bar_wait(tm_full + 8 * b, (n / 2) & 1, give))) break;
      tc_fence_after();
      const uint32_t from = tmem + b * kCols + ((uint32_t)(quarter * 32) << 16);
      auto leave_tile = [&]() {      // its room in tensor memory may be filled again
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (kPair) bar_arrive_cluster(first_of_pair(tm_empty + 8 * b));
          else bar_arrive(tm_empty + 8 * b);
        }
      };
      const int64_t part_words = (int64_t)kCols * S::kTileLanes;
      const uint32_t* parts = g.parts + (u - q.part) * part_words + rank * kLanes + in_tile;
      if (g.split > 1) {
        uint32_t* mine = g.parts + u * part_words + rank * kLanes + in_tile;
#pragma unroll 1
        for (int c = chunk0; c < cols; c += kNext) {
          uint32_t acc[32];
          tmem_load32(from + c, acc);
#pragma unroll
          for (int i = 0; i < 32; ++i) mine[(c + i) * S::kTileLanes] = acc[i];
        }
        leave_tile();
        if (!together()) break;
        if (warp == 2 && lane == 0) {
          uint32_t* seen = g.arrived + (u / g.split) * kBlocks + rank;
          __threadfence();      // stands between the block's parts, which this thread has seen to be written, and its count,
          const uint32_t before = atomicAdd(seen, 1u);
          if (before + 1 == (uint32_t)g.split) *seen = 0u;
          __threadfence();      // and between the others' counts and the block's reading of their parts
          words[2] = before + 1 == (uint32_t)g.split;
        }
        if (!together()) break;
        const bool last = words[2] != 0u;
        if (!together()) break;      // words[2] may change from here on
        if (!last) continue;
      }
#pragma unroll 1
      for (int c = chunk0; c < cols; c += kNext) {
        uint32_t acc[32];
        if (g.split == 1) {
          tmem_load32(from + c, acc);
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) acc[i] = __ldcg(parts + (c + i) * S::kTileLanes);
#pragma unroll 1
          for (int k = 1; k < g.split; ++k) {
            const uint32_t* next = parts + k * part_words;
            uint32_t w[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) w[i] = __ldcg(next + (c + i) * S::kTileLanes);
#pragma unroll
            for (int i = 0; i < 32; ++i)
              acc[i] = kInt8 ? acc[i] + w[i] : __float_as_uint(__uint_as_float(acc[i]) + __uint_as_float(w[i]));
          }
        }
        Ahead<kEpi> next;
        read(c + kNext, next);
        finish(c, ahead, acc);
        ahead = next;
      }
      if (g.split == 1) leave_tile();
    }
    __syncwarp();
  }
  // The other block's roles look at its own word.
  if (kPair && lane == 0 && words[1]) cluster_store(at_rank(smem_addr((const void*)(words + 1)), rank ^ 1), 1u);
  if (g.free_start) follow();
  auto all = [&]() {
    tc_fence_before();
    if (kPair) cluster_sync();
    else __syncthreads();
    tc_fence_after();
  };
  all();
  if (words[1]) {      // the same in both blocks of a pair by now: nothing may be on its way to their memory when they leave
    if (rank == 0 && lane == 0 && warp == 0) {
      const uint64_t t0 = now_ns();
      // Both blocks' copies report to this one's barriers.  Where one has asked for a stage and the other has not, the barrier is
      // told what to expect.
      const uint32_t mine = words[3], other = kPair ? cluster_load(at_rank(smem_addr((const void*)(words + 3)), 1)) : mine, most = max(mine, other);
      for (uint32_t k = most > (uint32_t)kStages ? most - kStages : 0; k < most; ++k) {
        const uint32_t bar = full + 8 * (k % kStages);
        if (k >= mine) bar_expect(bar, S::kStageBytes);
        else if (k >= other) bar_complete(bar, S::kStageBytes);
        bar_drain(bar, (k / kStages) & 1, t0);
      }
    }
    if (rank == 0 && warp == 1 && elect_one()) {
      tc_commit<kPair>(drain);
      bar_drain(drain, 0, now_ns());
    }
    all();
  }
  if (warp == 1) tmem_free<kPair>(tmem, kTmemCols);
}

}  // namespace mat
}  // namespace rtopk
