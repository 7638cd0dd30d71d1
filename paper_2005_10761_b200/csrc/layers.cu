// Host side of a worker's layers: linear layers on 4-bit codes, dropout and layer normalisation.
#include "matrix_host.cuh"

#include <cmath>

#include "micro.cuh"
#include "norm.cuh"

using namespace rtopk::mat;

namespace {

// Kernels get their shared memory at a context's first call of their family: each is loaded for that, which took a program's first context 17 ms
// for all of them, also where it only codes or orthogonalises.
enum Family : uint32_t { MICRO = 1, NORM = 2, NORM_BACK = NORM << 4 };      // of the normalisation, four each: by type and by what is read
template <class F>
int allow_once(rtopk_matrix* ctx, uint32_t family, F allow) {
  if (ctx->allowed & family) return RTOPK_OK;
  MAT_CUDA(allow());
  ctx->allowed |= family;
  return RTOPK_OK;
}
template <class T>
constexpr uint32_t norm_family(Family first, bool second) { return first << (2 * (sizeof(T) == 2) + second); }

// ----------------------------------------------------------------------------- 4-bit codes
int64_t micro_ld(int64_t cols) { return up(ceil_div(cols, 2), 16); }                                  // bytes of a row of codes, at least
int64_t micro_scale_bytes(int64_t rows, int64_t cols) { return ceil_div(rows, 128) * ceil_div(cols, 256) * 1024; }

struct MicroScratch {
  MicroOut x_rows, dy_rows, x_cols, dy_cols;
  MicroScratch(Carve& c, int64_t tokens, int64_t n_out, int64_t n_in) {
    c.take<char>(kPartsBytes);
    auto codes = [&](int64_t rows, int64_t cols) {
      MicroOut o;
      o.ld = up(ceil_div(cols, 2), 128);
      o.codes = c.take<uint8_t>(rows * o.ld);
      o.scales = c.take<uint8_t>(micro_scale_bytes(rows, cols));
      return o;
    };
    tokens = std::max<int64_t>(tokens, 1);
    x_rows = codes(tokens, n_in);
    dy_rows = codes(tokens, n_out);
    x_cols = codes(n_in, tokens);
    dy_cols = codes(n_out, tokens);
  }
};

template <class T>
CodeJob<T> code_job(const T* src, int64_t ld, int64_t rows, int64_t cols, const MicroOut& by_row, const MicroOut& by_col) {
  return {src, ld, (int)rows, (int)cols, rows_aligned(src, sizeof(T), 1, ld, 0, 16) ? 1 : 0, (int)ceil_div(cols, 128), by_row, by_col};
}
template <class T>
int64_t code_tiles(const CodeJob<T>& j) { return j.tiles_c * ceil_div(j.rows, 128); }

template <bool kRows, bool kColumns, bool kTile, class T>
int micro_code(rtopk_matrix* ctx, cudaStream_t st, const CodeJob<T>& job, const CodeJob<T>* second = nullptr) {
  const int64_t tiles = code_tiles(job), all = tiles + (second ? code_tiles(*second) : 0);
  if (job.vec && (!second || second->vec)) return launch(ctx, k_micro_code<T, kRows, kColumns, kTile, true>, dim3((unsigned)all), 256, 0, st, job, second ? *second : job, tiles);
  return launch(ctx, k_micro_code<T, kRows, kColumns, kTile, false>, dim3((unsigned)all), 256, 0, st, job, second ? *second : job, tiles);
}

// out[r][c] = sum over the contraction of row r of `rows` and row c of `cols`.  Results whose rows start on multiples of 32 bytes are written
// along the rows by threads that have a row each, where there are rows enough to fill tiles of 128; else along the lanes, which
// are the result's columns then.  early: `cols` is older than the launch before.
int micro_gemm(rtopk_matrix* ctx, bool early, bool free_start, const MicroOut& row, int64_t rows, const MicroOut& col, int64_t cols, int64_t depth, void* out, int bf16, int64_t ld_out,
               cudaStream_t st) {
  Gemm g = {};
  const int64_t bytes = ceil_div(depth, 2);
  g.depth = (int)bytes, g.batch = 1;
  g.out = out, g.out_bf16 = bf16;
  g.free_start = free_start;
  const Operand r = {row.codes, bytes, rows, row.ld, 0, row.scales}, c = {col.codes, bytes, cols, col.ld, 0, col.scales};
  if (rows > 64 && rows_aligned(out, bf16 ? 2 : 4, 1, ld_out, 0, 32)) {
    g.lanes = (int)rows, g.cols = (int)cols;
    g.out_col = 1, g.out_lane = ld_out;
    return gemm<EPI_MICRO_ROWS>(ctx, r, c, g, st);
  }
  g.lanes = (int)cols, g.cols = (int)rows;
  g.out_col = ld_out, g.out_lane = 1;
  g.p_early = early;
  return gemm<EPI_MICRO>(ctx, c, r, g, st);
}

bool bad_micro(const void* codes, int64_t ld, const void* scales, int64_t cols) {
  return !codes || !scales || !aligned_to(codes, 16) || !aligned_to(scales, 16) || ld < micro_ld(cols) || ld % 16;
}
MicroOut as_micro(const uint8_t* codes, int64_t ld, const uint8_t* scales) { return {const_cast<uint8_t*>(codes), const_cast<uint8_t*>(scales), ld}; }

int check_micro(const rtopk_matrix* ctx, int64_t tokens, int64_t n_out, int64_t n_in) {
  if (!ctx || tokens < 0 || n_out < 1 || n_in < 1 || tokens > kDimMax || n_out > kDimMax || n_in > kDimMax) return RTOPK_ERR_INVALID_ARG;
  return RTOPK_OK;
}
// Blocks of a coding launch are counted in 31 bits.
bool micro_too_large(int64_t rows, int64_t cols) { return ceil_div(rows, 128) * ceil_div(cols, 128) > INT32_MAX; }

template <class T>
int micro_weights(rtopk_matrix* ctx, const T* w, int64_t ld, int64_t n_out, int64_t n_in, int tile, const MicroOut& rows, const MicroOut& cols, cudaStream_t st) {
  const CodeJob<T> job = code_job(w, ld, n_out, n_in, rows, cols);
  if (tile == 1) return micro_code<true, false, false>(ctx, st, job);
  if (!cols.codes) return micro_code<true, false, true>(ctx, st, job);
  return micro_code<true, true, true>(ctx, st, job);
}

constexpr int kFewSmem = 96 * 1024;
template <class T, int kTokens>
int micro_few(rtopk_matrix* ctx, const T* x, int64_t ld_x, const MicroOut& w, int64_t tokens, int64_t n_out, int64_t n_in, T* out, int64_t ld_out, cudaStream_t st) {
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(n_out, 128) * 4, 2 * ctx->sms));
  return launch(ctx, k_micro_few<T, kTokens>, grid, 256, few_smem(kTokens, n_in), st, x, ld_x, rows_aligned(x, sizeof(T), 1, ld_x, 0, 16) ? 1 : 0, w, tokens, n_out, n_in, out, ld_out);
}

cudaError_t allow_micro() {
  auto few = [](auto kernel) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem); };
  for (const cudaError_t e : {few(k_micro_few<float, 1>), few(k_micro_few<float, 2>), few(k_micro_few<float, 4>), few(k_micro_few<__nv_bfloat16, 1>), few(k_micro_few<__nv_bfloat16, 2>),
                              few(k_micro_few<__nv_bfloat16, 4>), allow_smem<EPI_MICRO>(), allow_smem<EPI_MICRO_ROWS>()})
    if (e != cudaSuccess) return e;
  return cudaSuccess;
}

template <class T>
int micro_product(rtopk_matrix* ctx, const T* x, int64_t ld_x, const MicroOut& w, int64_t tokens, int64_t n_out, int64_t n_in, T* out, int64_t ld_out, cudaStream_t st) {
  // One launch, but its dot products take longer than reading W with several tokens: 4 through 4096 -> 4096 7.4 us against 8.9 of the product
  // kernel, 2 through 8192 -> 8192 17.3 against 16.5, 4 23.6.
  if ((tokens == 1 || (tokens <= kFewTokens && tokens * n_in * n_out <= 100000000)) && few_smem(tokens <= 2 ? (int)tokens : 4, n_in) <= kFewSmem) {
    if (tokens == 1) return micro_few<T, 1>(ctx, x, ld_x, w, tokens, n_out, n_in, out, ld_out, st);
    if (tokens == 2) return micro_few<T, 2>(ctx, x, ld_x, w, tokens, n_out, n_in, out, ld_out, st);
    return micro_few<T, 4>(ctx, x, ld_x, w, tokens, n_out, n_in, out, ld_out, st);
  }
  Carve c{ctx->scratch};
  MicroScratch s(c, tokens, n_out, n_in);
  MAT_TRY((micro_code<true, false, false>(ctx, st, code_job(x, ld_x, tokens, n_in, s.x_rows, MicroOut{}))));
  return micro_gemm(ctx, true, false, s.x_rows, tokens, w, n_out, n_in, out, sizeof(T) == 2, ld_out, st);
}

template <class T>
int micro_gradients(rtopk_matrix* ctx, const T* dy, int64_t ld_dy, const T* x, int64_t ld_x, const MicroOut& w_t, int64_t tokens, int64_t n_out, int64_t n_in, T* dx, int64_t ld_dx,
                    void* dw, int dw_bf16, int64_t ld_dw, cudaStream_t st) {
  Carve c{ctx->scratch};
  MicroScratch s(c, tokens, n_out, n_in);
  const CodeJob<T> dy_job = code_job(dy, ld_dy, tokens, n_out, dx ? s.dy_rows : MicroOut{}, dw ? s.dy_cols : MicroOut{});
  if (dw) {      // both in one launch
    const CodeJob<T> x_job = code_job(x, ld_x, tokens, n_in, MicroOut{}, s.x_cols);
    if (dx) MAT_TRY((micro_code<true, true, false>(ctx, st, dy_job, &x_job)));
    else MAT_TRY((micro_code<false, true, false>(ctx, st, dy_job, &x_job)));
  } else {
    MAT_TRY((micro_code<true, false, false>(ctx, st, dy_job)));
  }
  if (dx) MAT_TRY(micro_gemm(ctx, true, false, s.dy_rows, tokens, w_t, n_in, n_out, dx, sizeof(T) == 2, ld_dx, st));
  // The second product does not depend on the first and starts as SMs fall free.
  if (dw) MAT_TRY(micro_gemm(ctx, false, dx != nullptr, s.dy_cols, n_out, s.x_cols, n_in, tokens, dw, dw_bf16, ld_dw, st));
  return RTOPK_OK;
}

// ----------------------------------------------------------------------------- dropout and layer normalisation
// false: not a mask
bool as_mask(const rtopk_mask* m, Mask* out) {
  *out = {};
  if (!m) return true;
  if (!(m->p >= 0.0 && m->p < 1.0) || m->worker > 65535u || m->site > 32767u || !aligned_to(m->step_ptr, 4)) return false;
  const double limit = std::min(std::nearbyint(m->p * 65536.0), 65535.0);
  out->limit = (uint32_t)limit;
  out->factor = (float)(65536.0 / (65536.0 - limit));
  for (uint32_t i = 0; i < 10; ++i) out->keys[2 * i] = (uint32_t)m->seed + i * 0x9E3779B9u, out->keys[2 * i + 1] = (uint32_t)(m->seed >> 32) + i * 0xBB67AE85u;
  out->tag = 0x80000000u | m->site << 16 | m->worker;
  out->step = m->step, out->step_ptr = m->step_ptr;
  return true;
}

// Rows of whole vectors of eight values.
bool whole_vectors(const void* p, int elem, int64_t cols, int64_t ld) { return !p || (cols % 8 == 0 && rows_aligned(p, elem, 1, ld, 0, 8 * elem)); }

int check_rows(const rtopk_matrix* ctx, int64_t rows, int64_t cols, int dtype) {
  return !ctx || rows < 0 || cols < 1 || rows > kDimMax || cols > kDimMax || bad_dtype(dtype) ? RTOPK_ERR_INVALID_ARG : RTOPK_OK;
}

template <class T>
int dropout(rtopk_matrix* ctx, const T* x, int64_t ld_x, int64_t rows, int64_t cols, const Mask& mask, T* out, int64_t ld_out, cudaStream_t st) {
  const bool vec = whole_vectors(x, sizeof(T), cols, ld_x) && whole_vectors(out, sizeof(T), cols, ld_out);
  const int64_t units = ceil_div(cols, vec ? 8 : kWarpCols), per = vec ? 256 : 8;      // of four rows: threads or warps; of a block
  const DropoutGrid f(rows, units, per);
  if (f.bands > 65535) return RTOPK_ERR_UNSUPPORTED;
  return launch(ctx, vec ? k_dropout<T, true> : k_dropout<T, false>, dim3((unsigned)f.blocks, (unsigned)f.bands), 256, 0, st, x, ld_x, rows, cols, f.band, divisor((uint32_t)units), mask, out, ld_out);
}

// How a block takes rows: `warps` warps for each, `keep` pieces of 256 columns a warp, `rows_per` rows at a time.  Two pieces, so that what is
// done once a row is shared by 16 columns of a thread (many rows of one piece get two as well, the second empty); one where there are too few
// rows to fill the SMs, four where two do not reach.  Without alignment the next row waits in registers, which four pieces would not leave.
constexpr int kRowBlocks = 160;
struct RowSplit {
  int warps, rows_per, keep;
  int64_t blocks;
  bool fits, full;
  RowSplit(int sms, int64_t rows, int64_t cols, int most, bool vec) {      // most: pieces a warp, at most
    const int64_t pieces = ceil_div(cols, kWarpCols);
    fits = pieces <= kRowWarps * (vec ? most : 2);
    if (!fits) return;
    keep = pieces > 2 * kRowWarps ? 4 : pieces > kRowWarps || rows * pieces > sms * kRowWarps ? 2 : 1;
    warps = (int)ceil_div(pieces, keep);
    full = vec && cols == (int64_t)warps * keep * kWarpCols;
    rows_per = (int)std::min<int64_t>(kRowWarps / warps, ceil_div(rows, sms));
    blocks = std::min<int64_t>(std::min(sms, kRowBlocks), ceil_div(rows, rows_per));
  }
};

// Calls go(kVec, kFull, kKeep) with constants.
template <class T, int kMost, class F>
int row_variant(const RowSplit& f, bool vec, F go) {
  using yes = std::true_type;
  using no = std::false_type;
  auto with = [&](auto keep) { return f.full ? go(yes{}, yes{}, keep) : vec ? go(yes{}, no{}, keep) : go(no{}, no{}, keep); };
  if (f.keep == 1) return with(std::integral_constant<int, 1>{});
  if (f.keep == 2) return with(std::integral_constant<int, 2>{});
  if constexpr (kMost == 4) {
    const std::integral_constant<int, 4> keep;
    return f.full ? go(yes{}, yes{}, keep) : go(yes{}, no{}, keep);
  }
  return RTOPK_ERR_INTERNAL;
}
// For every variant with up to kMost pieces a warp.
template <class T, int kMost, class F>
cudaError_t allow_rows(F kernel_of) {
  cudaError_t worst = cudaSuccess;
  for (const int keep : {1, 2, 4})
    for (const int kind : {0, 1, 2}) {      // without alignment, with it, full rows
      if (keep > (kind ? kMost : 2)) continue;
      RowSplit f(1, 1, 1, 4, true);
      f.keep = keep, f.full = kind == 2;
      row_variant<T, kMost>(f, kind > 0, [&](auto v, auto full, auto k) {
        const cudaError_t e = cudaFuncSetAttribute(kernel_of(v, full, k), cudaFuncAttributeMaxDynamicSharedMemorySize, kRowSmem);
        if (e != cudaSuccess) worst = e;
        return RTOPK_OK;
      });
    }
  return worst;
}

template <class T, bool kResidual>
int norm_rows(rtopk_matrix* ctx, const NormArgs<T>& a, const RowSplit& f, bool vec, cudaStream_t st) {
  auto kernel_of = [](auto v, auto full, auto keep) { return k_layer_norm_rows<T, v, full, keep, kResidual>; };
  MAT_TRY(allow_once(ctx, norm_family<T>(NORM, kResidual), [&] { return allow_rows<T, 4>(kernel_of); }));
  return row_variant<T, 4>(f, vec, [&](auto v, auto full, auto keep) {
    return launch(ctx, kernel_of(v, full, keep), dim3((unsigned)f.blocks), 32 * f.warps * f.rows_per, RowShape<T, v, keep, kResidual ? 2 : 1>::kSmem, st, a, f.warps,
                  f.rows_per);
  });
}
template <class T>
int layer_norm(rtopk_matrix* ctx, const NormArgs<T>& a, bool vec, cudaStream_t st) {
  const RowSplit f(ctx->sms, a.rows, a.cols, 4, vec);
  if (f.fits) return a.residual ? norm_rows<T, true>(ctx, a, f, vec, st) : norm_rows<T, false>(ctx, a, f, vec, st);
  return launch(ctx, vec ? k_layer_norm_long<T, true> : k_layer_norm_long<T, false>, dim3((unsigned)a.rows), 32 * kRowWarps, 0, st, a);
}

// The columns' sums of a block's groups meet in its shared memory.
template <class T, bool kVec, int kKeep, bool kMore>
constexpr int kBackSmem = std::max(RowShape<T, kVec, kKeep, kMore ? 3 : 2>::kSmem, 2 * kRowWarps * kWarpCols * kKeep * 4);
template <class T>
constexpr int kBackMost = sizeof(T) == 2 ? 4 : 2;      // pieces a warp
template <class T, bool kMore>
int back_rows(rtopk_matrix* ctx, const NormBackArgs<T>& a, const RowSplit& f, bool vec, float* parts, cudaStream_t st) {
  auto kernel_of = [](auto v, auto full, auto keep) { return k_layer_norm_back_rows<T, v, full, keep, kMore>; };
  MAT_TRY(allow_once(ctx, norm_family<T>(NORM_BACK, kMore), [&] { return allow_rows<T, kBackMost<T>>(kernel_of); }));
  return row_variant<T, kBackMost<T>>(f, vec, [&](auto v, auto full, auto keep) {
    return launch(ctx, kernel_of(v, full, keep), dim3((unsigned)f.blocks), 32 * f.warps * f.rows_per, kBackSmem<T, v, keep, kMore>, st, a, f.warps, f.rows_per, parts);
  });
}

// Ranges of rows whose column sums are formed apart: four blocks for each of 148 SMs, but no fewer than 32 rows each.
int64_t norm_parts(int64_t rows, int64_t cols) { return std::max<int64_t>(1, std::min(ceil_div(rows, 32), 592 / ceil_div(cols, kWarpCols))); }

struct NormScratch {
  float* parts;
  NormScratch(Carve& c, int64_t rows, int64_t cols) { parts = c.take<float>(std::max(norm_parts(rows, cols), cols <= 4 * kRowWarps * kWarpCols ? std::min<int64_t>(rows, kRowBlocks) : 0) * 2 * cols); }
};

template <class T>
int layer_norm_gradients(rtopk_matrix* ctx, const NormBackArgs<T>& a, float* dgamma, float* dbeta, bool vec, cudaStream_t st) {
  Carve c{ctx->scratch};
  float* parts = dgamma || dbeta ? NormScratch(c, a.rows, a.cols).parts : nullptr;
  auto join = [&](int64_t count) { return launch(ctx, k_norm_join, dim3((unsigned)ceil_div(2 * (int64_t)a.cols, 32)), 32 * kJoinSlices, 0, st, parts, count, a.cols, dgamma, dbeta); };
  const RowSplit f(ctx->sms, a.rows, a.cols, kBackMost<T>, vec);
  if (f.fits) {
    MAT_TRY((a.dtotal ? back_rows<T, true>(ctx, a, f, vec, parts, st) : back_rows<T, false>(ctx, a, f, vec, parts, st)));
    return parts ? join(f.blocks) : RTOPK_OK;
  }
  if (parts) {      // first: the gradients may be written over what they are made of
    const int per = (int)ceil_div(a.rows, norm_parts(a.rows, a.cols));
    const int64_t count = ceil_div(a.rows, per);
    MAT_TRY(launch(ctx, vec ? k_norm_columns<T, true> : k_norm_columns<T, false>, dim3((unsigned)ceil_div(a.cols, kWarpCols), (unsigned)count), 256, 0, st, a.dy, a.ld_dy, a.total, a.ld_t,
                   a.mean, a.rstd, a.rows, a.cols, per, parts));
    MAT_TRY(join(count));
  }
  if (!a.dresidual && !a.dx) return RTOPK_OK;
  return launch(ctx, vec ? k_layer_norm_back_long<T, true> : k_layer_norm_back_long<T, false>, dim3((unsigned)a.rows), 32 * kRowWarps, 0, st, a);
}

}  // namespace

extern "C" {

int rtopk_micro_layout(int64_t rows, int64_t cols, int64_t* ld, int64_t* scale_bytes) {
  if (rows < 1 || cols < 1 || rows > kDimMax || cols > kDimMax) return RTOPK_ERR_INVALID_ARG;
  if (ld) *ld = micro_ld(cols);
  if (scale_bytes) *scale_bytes = micro_scale_bytes(rows, cols);
  return RTOPK_OK;
}

int rtopk_micro_weights(rtopk_matrix* ctx, const void* weights, int dtype, int64_t ld_w, int64_t n_out, int64_t n_in, int tile, uint8_t* codes, int64_t ld_codes, uint8_t* scales,
                        uint8_t* codes_t, int64_t ld_t, uint8_t* scales_t, void* stream) {
  MAT_TRY(check_micro(ctx, 0, n_out, n_in));
  if (bad_dtype(dtype) || bad_view(weights, elem(dtype), 1, n_out, n_in, ld_w, 0) || bad_micro(codes, ld_codes, scales, n_in) || (tile != 1 && tile != 32) ||
      (codes_t && (tile != 32 || bad_micro(codes_t, ld_t, scales_t, n_out))))
    return RTOPK_ERR_INVALID_ARG;
  if (micro_too_large(n_out, n_in)) return RTOPK_ERR_UNSUPPORTED;
  OnDevice on(ctx->device);
  if (!on.ok) return fail(ctx, cudaErrorInvalidDevice);
  const MicroOut rows = as_micro(codes, ld_codes, scales), cols = as_micro(codes_t, ld_t, scales_t);
  if (dtype == RTOPK_F32) return micro_weights(ctx, (const float*)weights, ld_w, n_out, n_in, tile, rows, cols, (cudaStream_t)stream);
  return micro_weights(ctx, (const __nv_bfloat16*)weights, ld_w, n_out, n_in, tile, rows, cols, (cudaStream_t)stream);
}

int rtopk_micro_scratch(int64_t tokens, int64_t n_out, int64_t n_in, int64_t* bytes) {
  if (!bytes || tokens < 0 || n_out < 1 || n_in < 1 || tokens > kDimMax || n_out > kDimMax || n_in > kDimMax) return RTOPK_ERR_INVALID_ARG;
  Carve c{nullptr};
  MicroScratch s(c, tokens, n_out, n_in);
  *bytes = c.at;
  return RTOPK_OK;
}

int rtopk_micro_product(rtopk_matrix* ctx, const void* x, int dtype, int64_t ld_x, const uint8_t* codes, int64_t ld_codes, const uint8_t* scales, int64_t tokens, int64_t n_out,
                        int64_t n_in, void* out, int64_t ld_out, void* stream) {
  MAT_TRY(check_micro(ctx, tokens, n_out, n_in));
  if (bad_dtype(dtype) || bad_micro(codes, ld_codes, scales, n_in)) return RTOPK_ERR_INVALID_ARG;
  if (tokens && (bad_view(x, elem(dtype), 1, tokens, n_in, ld_x, 0) || bad_view(out, elem(dtype), 1, tokens, n_out, ld_out, 0))) return RTOPK_ERR_INVALID_ARG;
  if (!tokens) return RTOPK_OK;
  if (micro_too_large(tokens, n_in)) return RTOPK_ERR_UNSUPPORTED;
  int64_t need = 0;
  rtopk_micro_scratch(tokens, n_out, n_in, &need);
  if (need > ctx->scratch_bytes) return RTOPK_ERR_INVALID_ARG;
  OnDevice on(ctx->device);
  if (!on.ok) return fail(ctx, cudaErrorInvalidDevice);
  MAT_TRY(allow_once(ctx, MICRO, allow_micro));
  const MicroOut w = as_micro(codes, ld_codes, scales);
  if (dtype == RTOPK_F32) return micro_product(ctx, (const float*)x, ld_x, w, tokens, n_out, n_in, (float*)out, ld_out, (cudaStream_t)stream);
  return micro_product(ctx, (const __nv_bfloat16*)x, ld_x, w, tokens, n_out, n_in, (__nv_bfloat16*)out, ld_out, (cudaStream_t)stream);
}

int rtopk_micro_gradients(rtopk_matrix* ctx, const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, int dtype, const uint8_t* codes_t, int64_t ld_t, const uint8_t* scales_t,
                          int64_t tokens, int64_t n_out, int64_t n_in, void* dx, int64_t ld_dx, void* dw, int dw_dtype, int64_t ld_dw, void* stream) {
  MAT_TRY(check_micro(ctx, tokens, n_out, n_in));
  if (bad_dtype(dtype) || (!dx && !dw) || (tokens && bad_view(dy, elem(dtype), 1, tokens, n_out, ld_dy, 0))) return RTOPK_ERR_INVALID_ARG;
  if (dx && ((tokens && bad_view(dx, elem(dtype), 1, tokens, n_in, ld_dx, 0)) || bad_micro(codes_t, ld_t, scales_t, n_out))) return RTOPK_ERR_INVALID_ARG;
  if (dw && (bad_dtype(dw_dtype) || bad_view(dw, elem(dw_dtype), 1, n_out, n_in, ld_dw, 0) || (tokens && bad_view(x, elem(dtype), 1, tokens, n_in, ld_x, 0))))
    return RTOPK_ERR_INVALID_ARG;
  if (micro_too_large(tokens, n_in + n_out + 128)) return RTOPK_ERR_UNSUPPORTED;
  int64_t need = 0;
  rtopk_micro_scratch(tokens, n_out, n_in, &need);
  if (tokens && need > ctx->scratch_bytes) return RTOPK_ERR_INVALID_ARG;
  OnDevice on(ctx->device);
  if (!on.ok) return fail(ctx, cudaErrorInvalidDevice);
  cudaStream_t st = (cudaStream_t)stream;
  if (!tokens) {      // an empty sum
    if (dw) MAT_CUDA(cudaMemset2DAsync(dw, ld_dw * elem(dw_dtype), 0, n_in * elem(dw_dtype), n_out, st));
    return RTOPK_OK;
  }
  MAT_TRY(allow_once(ctx, MICRO, allow_micro));
  const MicroOut w_t = as_micro(codes_t, ld_t, scales_t);
  if (dtype == RTOPK_F32)
    return micro_gradients(ctx, (const float*)dy, ld_dy, (const float*)x, ld_x, w_t, tokens, n_out, n_in, (float*)dx, ld_dx, dw, dw_dtype == RTOPK_BF16, ld_dw, st);
  return micro_gradients(ctx, (const __nv_bfloat16*)dy, ld_dy, (const __nv_bfloat16*)x, ld_x, w_t, tokens, n_out, n_in, (__nv_bfloat16*)dx, ld_dx, dw, dw_dtype == RTOPK_BF16, ld_dw, st);
}

int rtopk_dropout(rtopk_matrix* ctx, const void* x, int dtype, int64_t ld_x, int64_t rows, int64_t cols, const rtopk_mask* mask, void* out, int64_t ld_out, void* stream) {
  MAT_TRY(check_rows(ctx, rows, cols, dtype));
  Mask m;
  if (!mask || !as_mask(mask, &m)) return RTOPK_ERR_INVALID_ARG;
  if (!rows) return RTOPK_OK;
  if (bad_view(x, elem(dtype), 1, rows, cols, ld_x, 0) || bad_view(out, elem(dtype), 1, rows, cols, ld_out, 0)) return RTOPK_ERR_INVALID_ARG;
  OnDevice on(ctx->device);
  if (!on.ok) return fail(ctx, cudaErrorInvalidDevice);
  if (dtype == RTOPK_F32) return dropout(ctx, (const float*)x, ld_x, rows, cols, m, (float*)out, ld_out, (cudaStream_t)stream);
  return dropout(ctx, (const __nv_bfloat16*)x, ld_x, rows, cols, m, (__nv_bfloat16*)out, ld_out, (cudaStream_t)stream);
}

int rtopk_layer_norm(rtopk_matrix* ctx, const void* x, int64_t ld_x, const void* residual, int64_t ld_r, int dtype, int64_t rows, int64_t cols, const float* gamma, const float* beta,
                     float eps, const rtopk_mask* mask, void* out, int64_t ld_out, void* total, int64_t ld_t, float* mean, float* rstd, void* stream) {
  MAT_TRY(check_rows(ctx, rows, cols, dtype));
  Mask m;
  if (!as_mask(mask, &m) || !(eps >= 0.f) || !std::isfinite(eps) || !aligned_to(gamma, 4) || !aligned_to(beta, 4) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
    return RTOPK_ERR_INVALID_ARG;
  if (!rows) return RTOPK_OK;
  const size_t e = elem(dtype);
  if (bad_view(x, e, 1, rows, cols, ld_x, 0) || bad_view(out, e, 1, rows, cols, ld_out, 0) || (residual && bad_view(residual, e, 1, rows, cols, ld_r, 0)) ||
      (total && bad_view(total, e, 1, rows, cols, ld_t, 0)))
    return RTOPK_ERR_INVALID_ARG;
  OnDevice on(ctx->device);
  if (!on.ok) return fail(ctx, cudaErrorInvalidDevice);
  auto whole = [&](const void* p, int64_t ld) { return whole_vectors(p, e, cols, ld); };
  const bool vec = whole(x, ld_x) && whole(out, ld_out) && whole(residual, ld_r) && whole(total, ld_t) && aligned_to(gamma, 32) && aligned_to(beta, 32);
  auto go = [&](auto t) {
    using T = decltype(t);
    const NormArgs<T> a = {(const T*)x, (const T*)residual, (T*)out, (T*)total, ld_x, ld_r, ld_out, ld_t, gamma, beta, mean, rstd, (int)rows, (int)cols, eps, m};
    return layer_norm(ctx, a, vec, (cudaStream_t)stream);
  };
  return dtype == RTOPK_F32 ? go(float{}) : go(__nv_bfloat16{});
}

int rtopk_layer_norm_scratch(int64_t rows, int64_t cols, int64_t* bytes) {
  if (!bytes || rows < 0 || cols < 1 || rows > kDimMax || cols > kDimMax) return RTOPK_ERR_INVALID_ARG;
  Carve c{nullptr};
  NormScratch s(c, rows, cols);
  *bytes = c.at;
  return RTOPK_OK;
}

int rtopk_layer_norm_gradients(rtopk_matrix* ctx, const void* dy, int64_t ld_dy, const void* total, int64_t ld_t, const void* dtotal, int64_t ld_dt, int dtype, int64_t rows, int64_t cols,
                               const float* mean, const float* rstd, const float* gamma, const rtopk_mask* mask, void* dresidual, int64_t ld_dr, void* dx, int64_t ld_dx, float* dgamma,
                               float* dbeta, void* stream) {
  MAT_TRY(check_rows(ctx, rows, cols, dtype));
  Mask m;
  if (!as_mask(mask, &m) || (dx != nullptr) != (mask != nullptr) || (!dresidual && !dx && !dgamma && !dbeta) || !aligned_to(gamma, 4) || !aligned_to(dgamma, 4) || !aligned_to(dbeta, 4))
    return RTOPK_ERR_INVALID_ARG;
  const size_t e = elem(dtype);
  if (rows && (bad_view(dy, e, 1, rows, cols, ld_dy, 0) || bad_view(total, e, 1, rows, cols, ld_t, 0) || (dtotal && bad_view(dtotal, e, 1, rows, cols, ld_dt, 0)) || !mean || !rstd ||
               !aligned_to(mean, 4) || !aligned_to(rstd, 4) || (dresidual && bad_view(dresidual, e, 1, rows, cols, ld_dr, 0)) || (dx && bad_view(dx, e, 1, rows, cols, ld_dx, 0))))
    return RTOPK_ERR_INVALID_ARG;
  int64_t need = 0;
  rtopk_layer_norm_scratch(rows, cols, &need);
  if (rows && (dgamma || dbeta) && need > ctx->scratch_bytes) return RTOPK_ERR_INVALID_ARG;
  OnDevice on(ctx->device);
  if (!on.ok) return fail(ctx, cudaErrorInvalidDevice);
  cudaStream_t st = (cudaStream_t)stream;
  if (!rows) {      // empty sums
    if (dgamma) MAT_CUDA(cudaMemsetAsync(dgamma, 0, cols * sizeof(float), st));
    if (dbeta) MAT_CUDA(cudaMemsetAsync(dbeta, 0, cols * sizeof(float), st));
    return RTOPK_OK;
  }
  auto whole = [&](const void* p, int64_t ld) { return whole_vectors(p, e, cols, ld); };
  const bool vec = whole(dy, ld_dy) && whole(total, ld_t) && whole(dtotal, ld_dt) && whole(dresidual, ld_dr) && whole(dx, ld_dx) && aligned_to(gamma, 32);
  auto go = [&](auto t) {
    using T = decltype(t);
    const NormBackArgs<T> a = {(const T*)dy, (const T*)total, (const T*)dtotal, (T*)dresidual, (T*)dx, ld_dy, ld_t, ld_dt, ld_dr, ld_dx, gamma, mean, rstd, (int)rows, (int)cols, m};
    return layer_norm_gradients(ctx, a, dgamma, dbeta, vec, st);
  };
  return dtype == RTOPK_F32 ? go(float{}) : go(__nv_bfloat16{});
}

}  // extern "C"
