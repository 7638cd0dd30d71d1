// What the host sides of the matrix operators share: the context, launches, tensor maps, the choice of the product kernel's tile, and
// checks of arguments.
#pragma once

#include "../../include/rtopk.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "gemm.cuh"
#include "grids.h"

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

struct rtopk_matrix {
  int device = 0, sms = 0;
  int last_cuda_error = 0;
  int64_t scratch_bytes = 0;
  char* scratch = nullptr;
  bool owns_scratch = false;
  uint32_t* error = nullptr;
  uint32_t* arrived = nullptr;      // of split products, beside the error word
  uint32_t* parts = nullptr;        // partial sums of split products, at the scratch's start
  EncodeTiled encode = nullptr;
  uint64_t launches = 0;
  int test_giveup = 0;              // RTOPK_MATRIX_OPT_TEST_GIVEUP
  uint32_t allowed = 0;             // which families of layers.cu have their shared memory
};

namespace rtopk {
namespace mat {

inline int fail(rtopk_matrix* ctx, cudaError_t e) {
  ctx->last_cuda_error = (int)e;
  return RTOPK_ERR_CUDA;
}
#define MAT_CUDA(call)                                  \
  do {                                                  \
    cudaError_t e__ = (call);                           \
    if (e__ != cudaSuccess) return fail(ctx, e__);      \
  } while (0)
#define MAT_TRY(call)                                   \
  do {                                                  \
    const int s__ = (call);                             \
    if (s__ != RTOPK_OK) return s__;                    \
  } while (0)

struct OnDevice {
  int prev = -1;      // the device to go back to, if it is another one
  bool ok = true;
  explicit OnDevice(int dev) {
    int now = -1;
    if (cudaGetDevice(&now) != cudaSuccess) { ok = false; return; }
    if (now == dev) return;
    prev = now;
    ok = cudaSetDevice(dev) == cudaSuccess;
  }
  ~OnDevice() { if (prev >= 0) cudaSetDevice(prev); }
};

constexpr int64_t kDimMax = 1 << 30;
constexpr int64_t kBatchMax = 65535;
constexpr int64_t kDepthMax = 131072;     // 127 * 127 * depth stays below 2^31

static_assert(kPartBytes == kLanes * 256 * 4, "");
constexpr int kErrorBytes = 1024 + 2 * kSplitTiles * 4;

inline int64_t up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }
inline int64_t ceil_div(int64_t x, int64_t a) { return (x + a - 1) / a; }

// Divides the scratch; with base = null it only counts.
struct Carve {
  char* base;
  int64_t at = 0;
  template <class T>
  T* take(int64_t count) {
    T* p = base ? (T*)(base + at) : nullptr;
    at += up(count * (int64_t)sizeof(T), 1024);
    return p;
  }
};

// A kernel may start while the one before it in the stream ends; the kernels wait for it themselves.
template <class... P, class... A>
int launch_cluster(rtopk_matrix* ctx, int cluster, void (*kernel)(P...), dim3 grid, int threads, int smem, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  int n = 0;
  at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[n++].val.programmaticStreamSerializationAllowed = 1;
  if (cluster > 1) {
    at[n].id = cudaLaunchAttributeClusterDimension;
    at[n].val.clusterDim.x = cluster, at[n].val.clusterDim.y = at[n].val.clusterDim.z = 1;
    ++n;
  }
  cfg.attrs = at;
  cfg.numAttrs = n;
  MAT_CUDA(cudaLaunchKernelEx(&cfg, kernel, P(args)...));
  ++ctx->launches;
  return RTOPK_OK;
}
template <class... P, class... A>
int launch(rtopk_matrix* ctx, void (*kernel)(P...), dim3 grid, int threads, int smem, cudaStream_t st, A... args) {
  return launch_cluster(ctx, 1, kernel, grid, threads, smem, st, args...);
}

// Tensor map of a [batch][rows][cols] array: boxes of box_rows rows of one 128-byte swizzle row.
inline int tensor_map(rtopk_matrix* ctx, CUtensorMap* map, const void* base, bool int8, int64_t cols, int64_t rows, int64_t batch, int64_t ld, int64_t stride, int box_rows) {
  const int64_t e = int8 ? 1 : 2;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)batch};
  const cuuint64_t strides[2] = {(cuuint64_t)(ld * e), (cuuint64_t)((batch > 1 ? stride : rows * ld) * e)};
  const cuuint32_t box[3] = {(cuuint32_t)(kDepthBytes / e), (cuuint32_t)box_rows, 1};
  const cuuint32_t step[3] = {1, 1, 1};
  const CUresult r = ctx->encode(map, int8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(base), dims, strides, box, step,
                                 CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? RTOPK_OK : fail(ctx, cudaErrorInvalidValue);
}

// As stored: rows of `cols` contiguous elements (4-bit codes: bytes); 4-bit codes have scales.
struct Operand { const void* p; int64_t cols, rows, ld, stride; const void* scales; };

// Of the scales of 4-bit codes: 1024 bytes for every 128 rows and 256 codes (kDepthBytes).
inline int scale_map(rtopk_matrix* ctx, CUtensorMap* map, const Operand& o) {
  const int64_t steps = ceil_div(o.cols, kDepthBytes);
  const cuuint64_t dims[3] = {256, (cuuint64_t)steps, (cuuint64_t)ceil_div(o.rows, kLanes)};
  const cuuint64_t strides[2] = {1024, (cuuint64_t)(steps * 1024)};
  const cuuint32_t box[3] = {256, 1, 1}, step[3] = {1, 1, 1};
  const CUresult r = ctx->encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<void*>(o.scales), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                 CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? RTOPK_OK : fail(ctx, cudaErrorInvalidValue);
}
inline int scale_maps(rtopk_matrix* ctx, ScaleMaps* s, const Operand& p, const Operand& q) {
  MAT_TRY(scale_map(ctx, &s->p, p));
  return scale_map(ctx, &s->q, q);
}
inline int scale_maps(rtopk_matrix*, NoScales*, const Operand&, const Operand&) { return RTOPK_OK; }

template <int kCols, bool kPair>
int64_t gemm_tiles(const Gemm& g) {
  using S = GemmShape<kCols, kPair>;
  const int tiles_l = (int)ceil_div(g.lanes, S::kTileLanes), tiles_c = (int)ceil_div(g.cols, kCols);
  if (!g.tri) return (int64_t)tiles_l * tiles_c;
  int64_t n = 0;
  for (int c = 0; c < tiles_c; ++c) n += tri_lane_tiles<kCols, S::kTileLanes>(tiles_l, c);
  return n;
}

template <int kCols, bool kPair, int kEpi>
int gemm_tile(rtopk_matrix* ctx, const Operand& p, const Operand& q, Gemm g, int split, cudaStream_t st) {
  using S = GemmShape<kCols, kPair, is_micro(kEpi)>;
  constexpr bool kBytes = kEpi == EPI_CODED || is_micro(kEpi);
  constexpr bool kMnMajor = kEpi == EPI_APPLY || kEpi == EPI_OUT || kEpi == EPI_UPDATE;
  constexpr int kBlocks = kPair ? 2 : 1;
  g.tiles_l = (int)ceil_div(g.lanes, S::kTileLanes), g.tiles_c = (int)ceil_div(g.cols, kCols);
  g.tiles = (int)gemm_tiles<kCols, kPair>(g);
  if (!parts_fit((int64_t)g.tiles * g.batch, split, (int64_t)S::kTileLanes * kCols * 4)) return RTOPK_ERR_INTERNAL;      // the kernel would write past both
  g.split = split;
  g.test_giveup = ctx->test_giveup;
  if (split > 1) g.free_start = 0;      // the parts' room is the context's
  g.parts = ctx->parts, g.arrived = ctx->arrived, g.error = ctx->error;
  CUtensorMap mp, mq;
  MAT_TRY(tensor_map(ctx, &mp, p.p, kBytes, p.cols, p.rows, g.batch, p.ld, p.stride, kMnMajor ? 64 : kLanes));
  MAT_TRY(tensor_map(ctx, &mq, q.p, kBytes, q.cols, q.rows, g.batch, q.ld, q.stride, S::kQRows));
  Scales<kEpi> scales;
  MAT_TRY(scale_maps(ctx, &scales, p, q));
  const int grid = kBlocks * (int)std::min<int64_t>((int64_t)g.tiles * g.batch * split, ctx->sms / kBlocks);
  return launch_cluster(ctx, kBlocks, k_gemm<kCols, kPair, kEpi>, dim3(grid), kGemmThreads, S::kSmem, st, mp, mq, scales, g);
}

// Which tile, and in how many parts: the one for which this estimate of the time, in cycles, is least.  A step of 128 bytes of
// the contraction index takes the tensor core's time or what its stage needs from L2 (64 bytes a cycle and SM, measured);
// the results of a tile take so many cycles a column after the last products, six tenths of that beside the next tile's; parts
// are written and read again.  Where the choice is close: the products with X of 2048 x 2048 as two 128-column tiles a pair or one
// of 256, 257 and 258 us the whole operator; of four 1500 x 6000, eight tiles of 256 or sixteen of 128, 1350 and 1420 us.
//
// 4-bit codes have figures of their own: their steps hold twice the codes, their results no factors.  Fitted to 140 shapes from 9 x 256 -> 256 to
// 8192 x 4096 -> 8192 in every tile and up to four parts: the choice is 1.4 % slower than the best on average.
// They have no pair of 128 columns: of 63 such shapes and types it was the fastest for three, by 1.1 % at most, and mostly far behind
// (8192 x 8192 -> 8192, bfloat16: 234 us, in 192 columns 206).  And in a trial build with tiles forced one of them did not come to its end
// (5534 tokens, 3325 -> 6256, binary32), for a cause that is not known; another trial's did.
//
// Contractions beyond kStepsMax steps are cut further, as far as their parts fit the scratch, in several waves if need be: the tensor core
// drops what falls below its accumulator's last bit, which in 4096 instructions takes up to 2.5e-4 of a sum of equal terms; the
// parts are added with rounding.  One step of two nearly equal rows of 2^24 numbers: error 6.7e-3 in eight parts, 5.4e-4 in 256, as
// for short rows.
constexpr int64_t kStepsMax = 1024;
// The widest tile.  The scales of 4-bit codes need their place in tensor memory beside the accumulators.
template <int kEpi>
constexpr int kWidest = is_micro(kEpi) ? 192 : 256;
template <int kEpi>
int gemm(rtopk_matrix* ctx, const Operand& p, const Operand& q, const Gemm& g, cudaStream_t st) {
  constexpr bool kMicro = is_micro(kEpi);
  constexpr double kColumn = kEpi == EPI_CODED ? 35 : kEpi == EPI_GRAM ? 45 : 75;
  const int64_t steps = ceil_div((int64_t)g.depth * (kEpi == EPI_CODED || kMicro ? 1 : 2), kDepthBytes);
  const double column = g.out_bf16 ? 10 : 17;      // of 4-bit products
  double best = 1e300;
  int which = 0, parts = 1;
  auto consider = [&](int id, int64_t tiles, int cols, int blocks, int stage_bytes) {
    const int64_t sms = std::min(ctx->sms, kPartBlocks) / blocks, all = tiles * g.batch;
    const int64_t room = kPartsBytes / ((int64_t)cols * kLanes * blocks * 4), least = std::min(ceil_div(steps, kStepsMax), std::max<int64_t>(1, room / all));
    for (int split = (int)least; split <= std::max<int64_t>(8, least); ++split) {
      if (split > 1 && ((split > least && all * split > sms) || steps < 4 * split || !parts_fit(all, split, (int64_t)cols * kLanes * blocks * 4))) break;
      if ((split - 1) * ceil_div(steps, split) >= steps) continue;      // a part without any step
      const int64_t waves = ceil_div(all * split, sms);
      if (kMicro) {
        const double here = (double)std::min<int64_t>(cols, g.cols), pair = blocks - 1;
        const double main = (double)ceil_div(steps, split) * std::max(stage_bytes / 90.0, cols * 2.0) + 1000 * pair, tail = here * column;
        const double t = main + tail + (waves - 1) * std::max(main, 0.3 * tail) + 2000 * pair + (split > 1 ? here * (2.0 + 16.0 * split) + 6000 : 0);
        if (t < best) best = t, which = id, parts = split;
        continue;
      }
      const double main = (double)ceil_div(steps, split) * std::max(stage_bytes / 64.0, cols * 2.0) + 500, tail = cols * kColumn;
      const double t = main + tail + (waves - 1) * std::max(main, 0.6 * tail) + (split > 1 ? cols * (16.0 + 16.0 * split) + 3000 : 0);
      if (t < best) best = t, which = id, parts = split;
    }
  };
  consider(0, gemm_tiles<64, false>(g), 64, 1, GemmShape<64, false, kMicro>::kStageBytes);
  consider(1, gemm_tiles<128, false>(g), 128, 1, GemmShape<128, false, kMicro>::kStageBytes);
  if constexpr (!kMicro) consider(2, gemm_tiles<128, true>(g), 128, 2, GemmShape<128, true, kMicro>::kStageBytes);
  consider(3, gemm_tiles<kWidest<kEpi>, true>(g), kWidest<kEpi>, 2, GemmShape<kWidest<kEpi>, true, kMicro>::kStageBytes);
  switch (which) {
    case 0: return gemm_tile<64, false, kEpi>(ctx, p, q, g, parts, st);
    case 1: return gemm_tile<128, false, kEpi>(ctx, p, q, g, parts, st);
    case 2:      // never chosen for 4-bit codes
      if constexpr (!kMicro) return gemm_tile<128, true, kEpi>(ctx, p, q, g, parts, st);
      [[fallthrough]];
    default: return gemm_tile<kWidest<kEpi>, true, kEpi>(ctx, p, q, g, parts, st);
  }
}

template <int kEpi>
cudaError_t allow_smem() {
  cudaError_t e = cudaFuncSetAttribute(k_gemm<64, false, kEpi>, cudaFuncAttributeMaxDynamicSharedMemorySize, GemmShape<64, false, is_micro(kEpi)>::kSmem);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(k_gemm<128, false, kEpi>, cudaFuncAttributeMaxDynamicSharedMemorySize, GemmShape<128, false, is_micro(kEpi)>::kSmem);
  if constexpr (!is_micro(kEpi))
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_gemm<128, true, kEpi>, cudaFuncAttributeMaxDynamicSharedMemorySize, GemmShape<128, true, is_micro(kEpi)>::kSmem);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(k_gemm<kWidest<kEpi>, true, kEpi>, cudaFuncAttributeMaxDynamicSharedMemorySize, GemmShape<kWidest<kEpi>, true, is_micro(kEpi)>::kSmem);
  return e;
}

inline bool aligned_to(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
// Rows that start on multiples of `bytes`, wherever in the batch.
inline bool rows_aligned(const void* p, size_t elem, int64_t batch, int64_t ld, int64_t stride, size_t bytes) {
  return aligned_to(p, bytes) && ld * elem % bytes == 0 && (batch == 1 || stride * elem % bytes == 0);
}

// Batches of matrices with `n` contiguous elements in rows `ld` apart.
inline bool bad_view(const void* p, size_t elem, int64_t batch, int64_t m, int64_t n, int64_t ld, int64_t stride) {
  return !p || !aligned_to(p, elem) || ld < n || (batch > 1 && stride < (m - 1) * ld + n);
}
inline bool bad_dtype(int t) { return t != RTOPK_F32 && t != RTOPK_BF16; }
inline size_t elem(int t) { return t == RTOPK_F32 ? 4 : 2; }

}  // namespace mat
}  // namespace rtopk
