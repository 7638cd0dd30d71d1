// Host side of the matrix operators: argument checks, the division of the scratch and the launch sequences.
// All device work is enqueued on the caller's stream; only the documented status read synchronises.
#include "matrix_host.cuh"

#include <cmath>
#include <new>

#include "coded.cuh"
#include "orthogonal.cuh"

using namespace rtopk::mat;

namespace {

struct OrthScratch {
  float* x;               // X in 32 bits; its 16-bit form is read by a product while the next one is written
  __half *hi[2], *gram, *poly;
  float *gram_d, *poly_d, *row_sums;
  double* part;
  int slots;
  int64_t ld_x, ld_a, stride_x, stride_a, stride_d;
  OrthScratch(Carve& c, int64_t batch, int64_t s, int64_t l) {
    ld_x = up(l, 64), ld_a = up(s, 64);
    stride_x = s * ld_x, stride_a = s * ld_a, stride_d = up(s, 64);
    c.take<char>(kPartsBytes);
    part = c.take<double>(batch * kNormBlocks);
    for (auto& h : hi) h = c.take<__half>(batch * stride_x);
    x = c.take<float>(batch * stride_x);
    gram = c.take<__half>(batch * stride_a);
    poly = c.take<__half>(batch * stride_a);
    gram_d = c.take<float>(batch * stride_d);
    poly_d = c.take<float>(batch * stride_d);
    slots = (int)ceil_div(l, 32);
    row_sums = c.take<float>(batch * slots * stride_d);
  }
};

// Sizes whose scratch would not fit 64 bits of bytes (nor any memory).
bool orth_too_large(int64_t batch, int64_t m, int64_t n) { return (double)batch * (double)std::min(m, n) * (double)up(std::max(m, n), 64) > 0x1p56; }

struct CodedScratch {
  int8_t *x_rows, *dy_rows, *x_cols, *dy_cols;
  float *x_row_s, *dy_row_s, *x_col_s, *dy_col_s;
  uint32_t* col_max;      // n_in, then n_out
  int64_t ld_in, ld_out, ld_tok;
  CodedScratch(Carve& c, int64_t tokens, int64_t n_out, int64_t n_in) {
    ld_in = up(n_in, 128), ld_out = up(n_out, 128), ld_tok = up(std::max<int64_t>(tokens, 1), 128);
    c.take<char>(kPartsBytes);
    x_rows = c.take<int8_t>(tokens * ld_in);
    dy_rows = c.take<int8_t>(tokens * ld_out);
    x_cols = c.take<int8_t>(n_in * ld_tok);
    dy_cols = c.take<int8_t>(n_out * ld_tok);
    x_row_s = c.take<float>(tokens);
    dy_row_s = c.take<float>(tokens);
    x_col_s = c.take<float>(n_in);
    dy_col_s = c.take<float>(n_out);
    col_max = c.take<uint32_t>(n_in + n_out);
  }
};

constexpr float kQuintic[3] = {3.4445f, -4.7750f, 2.0315f};

struct Target {
  int epi;                // EPI_OUT or EPI_UPDATE
  void* out;
  int bf16;
  int64_t ld, stride;
  float keep, rate;
};

int orthogonal_small(rtopk_matrix* ctx, Source src, const Target& to, int64_t batch, int64_t m, int64_t n, int steps, const float* coef, cudaStream_t st) {
  src.m = (int)m, src.n = (int)n;
  SmallOut o = {};
  o.w = to.epi == EPI_UPDATE ? (float*)to.out : nullptr;
  o.test_giveup = ctx->test_giveup;
  o.out = to.out, o.bf16 = to.bf16, o.ld = to.ld, o.stride = to.stride, o.keep = to.keep, o.rate = to.rate, o.steps = steps;
  for (int i = 0; i < 3 * steps; ++i) o.coef[i] = coef ? coef[i] : kQuintic[i % 3];
  const int64_t s = std::min(m, n), l = std::max(m, n);
  if (s > kSmall || l > kSmallLong) {
    int blocks = 1;
    while (blocks * kMidChunks * kSmall < l) blocks *= 2;
    return launch_cluster(ctx, blocks, k_orth_cluster, dim3((unsigned)(batch * blocks)), kMidThreads, kMidBytes, st, src, o, m > n ? 1 : 0,
                          (int)ceil_div(ceil_div(l, kSmall), blocks), ctx->error);
  }
  return launch(ctx, k_orth_small, dim3((unsigned)batch), kSmallThreads, small_bytes((int)std::max(m, n)), st, src, o, m > n ? 1 : 0, ctx->error);
}

int orthogonal(rtopk_matrix* ctx, Source src, const Target& to, int64_t batch, int64_t m, int64_t n, int steps, const float* coef, cudaStream_t st) {
  const int64_t s = std::min(m, n), l = std::max(m, n);
  const bool tall = m > n;
  Carve c{ctx->scratch};
  OrthScratch w(c, batch, s, l);
  if (c.at > ctx->scratch_bytes) return RTOPK_ERR_INVALID_ARG;
  // one launch: 1.6 times as fast as a chain at 128 x 256, 1.05 times at 128 x 1000 and 2048 (1.7 times for thirty of them);
  // beyond, X does not fit a cluster
  if ((s <= kSmall && l <= kSmallLong) || (s <= kMid && l <= kMidLong)) return orthogonal_small(ctx, src, to, batch, m, n, steps, coef, st);
  src.m = (int)m, src.n = (int)n;
  src.part = w.part;
  src.parts = (int)std::min<int64_t>(kNormBlocks, ceil_div(m * ceil_div(n, kNormSpan), 8));
  MAT_TRY(launch(ctx, k_norm, dim3(src.parts, (unsigned)batch), 256, 0, st, src));
  MAT_TRY(launch(ctx, k_split, dim3((unsigned)ceil_div(n, 64), (unsigned)ceil_div(m, 64), (unsigned)batch), 256, 0, st, src, w.x, w.hi[0], w.ld_x, w.stride_x,
                 w.row_sums, w.slots, w.stride_d, tall ? 1 : 0));
  int cur = 0;
  for (int i = 0; i < steps; ++i) {
    const float* k = coef ? coef + 3 * i : kQuintic;
    const Operand x = {w.hi[cur], l, s, w.ld_x, w.stride_x, nullptr};
    const Operand gram = {w.gram, s, s, w.ld_a, w.stride_a, nullptr}, poly = {w.poly, s, s, w.ld_a, w.stride_a, nullptr};
    Gemm g = {};
    g.batch = (int)batch;
    g.d_stride = w.stride_d;
    g.row_sums = w.row_sums, g.slots = w.slots;
    g.a = k[0], g.b = k[1], g.c = k[2];
    g.lanes = g.cols = (int)s, g.depth = (int)l, g.tri = 1;
    g.h = w.gram, g.ld = w.ld_a, g.stride = w.stride_a, g.d_out = w.gram_d;
    MAT_TRY(gemm<EPI_GRAM>(ctx, x, x, g, st));
    g.depth = (int)s;
    g.o = w.gram, g.d_in = w.gram_d, g.h = w.poly, g.d_out = w.poly_d;
    MAT_TRY(gemm<EPI_POLY>(ctx, gram, gram, g, st));
    g.lanes = (int)l, g.tri = 0;
    g.p_early = 1;      // the launch before wrote the polynomial, X is older
    g.x = w.x, g.ld = w.ld_x, g.stride = w.stride_x, g.d_in = w.poly_d;
    if (i + 1 < steps) {
      g.h = w.hi[cur ^ 1];
      MAT_TRY(gemm<EPI_APPLY>(ctx, x, poly, g, st));
      cur ^= 1;
    } else {
      g.out = to.out, g.out_bf16 = to.bf16, g.keep = to.keep, g.rate = to.rate;
      g.out_col = tall ? 1 : to.ld, g.out_lane = tall ? to.ld : 1, g.out_batch = to.stride;
      if (to.epi == EPI_OUT) MAT_TRY(gemm<EPI_OUT>(ctx, x, poly, g, st));
      else MAT_TRY(gemm<EPI_UPDATE>(ctx, x, poly, g, st));
    }
  }
  return RTOPK_OK;
}

int check_orth(const rtopk_matrix* ctx, int64_t batch, int64_t m, int64_t n, int steps, const float* coef, float eps) {
  if (!ctx || batch < 1 || m < 1 || n < 1 || m > kDimMax || n > kDimMax || steps < 1 || steps > 64) return RTOPK_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || !std::isfinite(eps)) return RTOPK_ERR_INVALID_ARG;
  if (coef)
    for (int i = 0; i < 3 * steps; ++i)
      if (!std::isfinite(coef[i])) return RTOPK_ERR_INVALID_ARG;
  if (batch > kBatchMax || m > 64 * kBatchMax || orth_too_large(batch, m, n)) return RTOPK_ERR_UNSUPPORTED;
  return RTOPK_OK;
}

// As many warps as hold a row in their registers, 4096 bytes each (8192 rows of 4096 bfloat16 values in two warps each 31 us, in one
// with twice the registers 38); up to eight where there are too few rows to fill the SMs (24 rows of 8192: 4.9 us, 6.9 in four).
template <class T>
int code_rows(rtopk_matrix* ctx, const T* src, int64_t ld, int64_t rows, int64_t cols, const float* mul, int8_t* codes, int64_t ld_codes, float* scales, cudaStream_t st,
              int64_t padded = 0, uint32_t* clear = nullptr, int64_t clear_words = 0) {
  const int vec = rows_aligned(src, sizeof(T), 1, ld, 0, 16), mul_vec = aligned_to(mul, 16);
  auto go = [&](auto kernel, auto kernel_mul, int warps) {
    return launch(ctx, mul ? kernel_mul : kernel, dim3((unsigned)ceil_div(rows, 8 / warps)), 256, 0, st, src, ld, rows, cols, vec, mul, mul_vec, codes, ld_codes,
                  std::max(cols, padded), scales, clear, clear_words);
  };
  const int64_t warps = rows <= 4 * ctx->sms ? ceil_div(cols, 256) : ceil_div(cols * sizeof(T), 4096);
  if (warps <= 1) return go(k_code_rows<T, 1, false>, k_code_rows<T, 1, true>, 1);
  if (warps <= 2) return go(k_code_rows<T, 2, false>, k_code_rows<T, 2, true>, 2);
  if (warps <= 4) return go(k_code_rows<T, 4, false>, k_code_rows<T, 4, true>, 4);
  return go(k_code_rows<T, 8, false>, k_code_rows<T, 8, true>, 8);
}

int coded_gemm(rtopk_matrix* ctx, bool lanes_early, bool free_start, const int8_t* lane_codes, int64_t ld_lane, const float* lane_scale, int64_t lanes, const int8_t* col_codes, int64_t ld_col,
               const float* col_scale, int64_t cols, int64_t depth, void* out, int bf16, int64_t ld_out, cudaStream_t st) {
  Gemm g = {};
  g.lanes = (int)lanes, g.cols = (int)cols, g.depth = (int)depth, g.batch = 1;
  g.out = out, g.out_bf16 = bf16, g.out_col = ld_out, g.out_lane = 1;
  g.scale_col = col_scale, g.scale_lane = lane_scale;
  g.p_early = lanes_early, g.free_start = free_start;
  return gemm<EPI_CODED>(ctx, {lane_codes, depth, lanes, ld_lane, 0, nullptr}, {col_codes, depth, cols, ld_col, 0, nullptr}, g, st);
}

bool bad_codes(const int8_t* p, int64_t ld, int64_t cols) { return !p || !aligned_to(p, 16) || ld < cols || ld % 16; }

int check_coded(const rtopk_matrix* ctx, int64_t tokens, int64_t n_out, int64_t n_in) {
  if (!ctx || tokens < 0 || n_out < 1 || n_in < 1 || tokens > kDimMax || n_out > kDimMax || n_in > kDimMax) return RTOPK_ERR_INVALID_ARG;
  return RTOPK_OK;
}

template <class T, int kTokens>
int product_few(rtopk_matrix* ctx, const T* x, int64_t ld_x, const int8_t* codes, int64_t ld_codes, const float* scales, int64_t tokens, int64_t n_out, int64_t n_in,
                T* out, int64_t ld_out, cudaStream_t st) {
  const int smem = kTokens * few_row((int)n_in);
  const int64_t fit = std::max<int64_t>(1, std::min<int64_t>(4, kSmemLimit / (smem + 2048)));
  const int grid = (int)std::min<int64_t>(ceil_div(n_out, 16), ctx->sms * fit);
  return launch(ctx, k_product_few<T, kTokens>, dim3(grid), kFewThreads, smem, st, x, ld_x, rows_aligned(x, sizeof(T), 1, ld_x, 0, 16) ? 1 : 0, codes, ld_codes, scales, tokens,
                n_out, n_in, out, ld_out);
}

template <class T>
int product(rtopk_matrix* ctx, const T* x, int64_t ld_x, const int8_t* codes, int64_t ld_codes, const float* scales, int64_t tokens, int64_t n_out, int64_t n_in,
            T* out, int64_t ld_out, cudaStream_t st) {
  // One launch saves 2 us over two, but its dot products take longer than reading W once there are many: 4 tokens through
  // 1500 -> 6000 6.9 us against 7.5, through 4096 -> 4096 9.2 against 7.4, through 8192 -> 8192 29.7 against 17.5.
  const int64_t few = tokens <= 1 ? 1 : tokens <= 2 ? 2 : 4;
  if (tokens <= 4 && few * few_row((int)n_in) <= kFewBytes && (tokens == 1 || tokens * n_in * n_out <= 40000000)) {
    if (few == 1) return product_few<T, 1>(ctx, x, ld_x, codes, ld_codes, scales, tokens, n_out, n_in, out, ld_out, st);
    if (few == 2) return product_few<T, 2>(ctx, x, ld_x, codes, ld_codes, scales, tokens, n_out, n_in, out, ld_out, st);
    return product_few<T, 4>(ctx, x, ld_x, codes, ld_codes, scales, tokens, n_out, n_in, out, ld_out, st);
  }
  Carve c{ctx->scratch};
  CodedScratch w(c, tokens, n_out, n_in);
  MAT_TRY(code_rows(ctx, x, ld_x, tokens, n_in, nullptr, w.x_rows, w.ld_in, w.x_row_s, st, w.ld_in));
  // 8 tokens through 4096 -> 4096 7.4 us, the product kernel 9.2 (both 17.5 through 8192 -> 8192); with 16 tokens the product
  // kernel is the faster one, 17.5 against 19.9.
  if (tokens <= 8)
    return launch(ctx, k_product_tokens<T>, dim3((unsigned)ceil_div(n_out, kTokChannels)), kTokThreads, 0, st, w.x_rows, w.ld_in, w.x_row_s, codes, ld_codes, scales, tokens, n_out,
                  n_in, out, ld_out);
  return coded_gemm(ctx, true, false, codes, ld_codes, scales, n_out, w.x_rows, w.ld_in, w.x_row_s, tokens, n_in, out, sizeof(T) == 2, ld_out, st);
}

template <class T>
int gradients(rtopk_matrix* ctx, const T* dy, int64_t ld_dy, const T* x, int64_t ld_x, const int8_t* codes_t, int64_t ld_t, const float* scales, int64_t tokens,
              int64_t n_out, int64_t n_in, T* dx, int64_t ld_dx, void* dw, int dw_dtype, int64_t ld_dw, cudaStream_t st) {
  Carve c{ctx->scratch};
  CodedScratch w(c, tokens, n_out, n_in);
  // All coding first, then both products: the second does not depend on the first and starts as SMs fall free.
  if (dx) MAT_TRY(code_rows(ctx, dy, ld_dy, tokens, n_out, scales, w.dy_rows, w.ld_out, w.dy_row_s, st, 0, w.col_max, dw ? n_in + n_out : 0));
  if (dw) {
    if (!dx) MAT_CUDA(cudaMemsetAsync(w.col_max, 0, (n_in + n_out) * sizeof(uint32_t), st));
    Columns<T> cx = {x, ld_x, (int)n_in, rows_aligned(x, sizeof(T), 1, ld_x, 0, 16), (int)ceil_div(n_in, 256), w.col_max, w.x_cols, w.x_col_s};
    Columns<T> cy = {dy, ld_dy, (int)n_out, rows_aligned(dy, sizeof(T), 1, ld_dy, 0, 16), (int)ceil_div(n_out, 256), w.col_max + n_in, w.dy_cols, w.dy_col_s};
    const int64_t across = cx.tiles + cy.tiles;
    const int per = (int)std::max<int64_t>(32, ceil_div(tokens, std::max<int64_t>(1, 6 * ctx->sms / across)));      // all blocks at once
    MAT_TRY(launch(ctx, k_col_max<T>, dim3((unsigned)across, (unsigned)ceil_div(tokens, per)), 256, 0, st, cx, cy, tokens, per));
    cx.tiles = (int)ceil_div(n_in, 64), cy.tiles = (int)ceil_div(n_out, 64);
    MAT_TRY(launch(ctx, k_code_cols<T>, dim3((unsigned)(cx.tiles + cy.tiles), (unsigned)ceil_div(tokens, 128)), 256, 0, st, cx, cy, tokens, w.ld_tok));
  }
  if (dx) MAT_TRY(coded_gemm(ctx, true, false, codes_t, ld_t, nullptr, n_in, w.dy_rows, w.ld_out, w.dy_row_s, tokens, n_out, dx, sizeof(T) == 2, ld_dx, st));
  if (dw)
    MAT_TRY(coded_gemm(ctx, false, dx != nullptr, w.x_cols, w.ld_tok, w.x_col_s, n_in, w.dy_cols, w.ld_tok, w.dy_col_s, n_out, tokens, dw, dw_dtype == RTOPK_BF16, ld_dw, st));
  return RTOPK_OK;
}

}  // namespace

extern "C" {

int rtopk_matrix_create(rtopk_matrix** out, int device, void* scratch, int64_t scratch_bytes, void* stream) {
  if (!out) return RTOPK_ERR_INVALID_ARG;
  *out = nullptr;
  if (scratch_bytes < 0 || device < 0 || !aligned_to(scratch, 256)) return RTOPK_ERR_INVALID_ARG;
  rtopk_matrix* ctx = new (std::nothrow) rtopk_matrix;
  if (!ctx) return RTOPK_ERR_ALLOC;
  ctx->device = device;
  ctx->scratch_bytes = scratch_bytes;
  OnDevice on(device);
  int status = on.ok ? RTOPK_OK : RTOPK_ERR_CUDA;
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (status == RTOPK_OK && (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
                             found != cudaDriverEntryPointSuccess || cudaDeviceGetAttribute(&ctx->sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess ||
                             allow_smem<EPI_GRAM>() != cudaSuccess || allow_smem<EPI_POLY>() != cudaSuccess || allow_smem<EPI_APPLY>() != cudaSuccess ||
                             allow_smem<EPI_OUT>() != cudaSuccess || allow_smem<EPI_UPDATE>() != cudaSuccess || allow_smem<EPI_CODED>() != cudaSuccess ||
                             cudaFuncSetAttribute(k_orth_small, cudaFuncAttributeMaxDynamicSharedMemorySize, small_bytes(kSmallLong)) != cudaSuccess ||
                             cudaFuncSetAttribute(k_orth_cluster, cudaFuncAttributeMaxDynamicSharedMemorySize, kMidBytes) != cudaSuccess))
    status = RTOPK_ERR_CUDA;
  ctx->encode = (EncodeTiled)fn;
  ctx->scratch = (char*)scratch;
  if (status == RTOPK_OK) {
    if (cudaMalloc(&ctx->error, kErrorBytes) != cudaSuccess) status = RTOPK_ERR_ALLOC;
    else if (cudaMemsetAsync(ctx->error, 0, kErrorBytes, (cudaStream_t)stream) != cudaSuccess) status = RTOPK_ERR_CUDA;
    else if (!scratch && scratch_bytes) {
      ctx->owns_scratch = cudaMalloc(&ctx->scratch, scratch_bytes) == cudaSuccess;
      if (!ctx->owns_scratch) status = RTOPK_ERR_ALLOC;
    }
  }
  if (status != RTOPK_OK) {
    cudaGetLastError();
    rtopk_matrix_destroy(ctx);
    return status;
  }
  ctx->arrived = ctx->error + 64;
  ctx->parts = (uint32_t*)ctx->scratch;
  *out = ctx;
  return RTOPK_OK;
}

int rtopk_matrix_destroy(rtopk_matrix* ctx) {
  if (!ctx) return RTOPK_OK;
  OnDevice on(ctx->device);
  if (ctx->owns_scratch) cudaFree(ctx->scratch);
  if (ctx->error) cudaFree(ctx->error);
  delete ctx;
  return RTOPK_OK;
}

int rtopk_matrix_set_option(rtopk_matrix* ctx, int option, int64_t value) {
  if (!ctx || option != RTOPK_MATRIX_OPT_TEST_GIVEUP || (value != 0 && value != 1)) return RTOPK_ERR_INVALID_ARG;
  ctx->test_giveup = (int)value;
  return RTOPK_OK;
}

int rtopk_matrix_last_cuda_error(const rtopk_matrix* ctx) { return ctx ? ctx->last_cuda_error : 0; }

int rtopk_matrix_get_launch_count(const rtopk_matrix* ctx, uint64_t* out) {
  if (!ctx || !out) return RTOPK_ERR_INVALID_ARG;
  *out = ctx->launches;
  return RTOPK_OK;
}

int rtopk_matrix_poll_status(rtopk_matrix* ctx, void* stream) {
  if (!ctx) return RTOPK_ERR_INVALID_ARG;
  OnDevice on(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  uint32_t e = 0;
  MAT_CUDA(cudaMemcpyAsync(&e, ctx->error, sizeof e, cudaMemcpyDeviceToHost, st));
  MAT_CUDA(cudaStreamSynchronize(st));
  if (!e) return RTOPK_OK;
  MAT_CUDA(cudaMemsetAsync(ctx->error, 0, kErrorBytes, st));      // the counters too: a block that gave up may have left them
  return RTOPK_ERR_INTERNAL;
}

int rtopk_orthogonalize_scratch(int64_t batch, int64_t m, int64_t n, int64_t* bytes) {
  if (!bytes || batch < 1 || m < 1 || n < 1 || batch > kBatchMax || m > kDimMax || n > kDimMax) return RTOPK_ERR_INVALID_ARG;
  if (orth_too_large(batch, m, n)) return RTOPK_ERR_UNSUPPORTED;
  Carve c{nullptr};
  OrthScratch w(c, batch, std::min(m, n), std::max(m, n));
  *bytes = c.at;
  return RTOPK_OK;
}

int rtopk_orthogonalize(rtopk_matrix* ctx, const void* src, int src_dtype, int64_t ld_src, int64_t stride_src, void* out, int out_dtype, int64_t ld_out,
                        int64_t stride_out, int64_t batch, int64_t m, int64_t n, int steps, const float* coef, float eps, void* stream) {
  MAT_TRY(check_orth(ctx, batch, m, n, steps, coef, eps));
  if (bad_dtype(src_dtype) || bad_dtype(out_dtype) || bad_view(src, elem(src_dtype), batch, m, n, ld_src, stride_src) ||
      bad_view(out, elem(out_dtype), batch, m, n, ld_out, stride_out))
    return RTOPK_ERR_INVALID_ARG;
  OnDevice on(ctx->device);
  if (!on.ok) return fail(ctx, cudaErrorInvalidDevice);
  Source s = {};
  s.src = src, s.bf16 = src_dtype == RTOPK_BF16, s.ld = ld_src, s.stride = stride_src, s.eps = eps;
  s.vec = rows_aligned(src, elem(src_dtype), batch, ld_src, stride_src, 4 * elem(src_dtype));
  const Target to = {EPI_OUT, out, out_dtype == RTOPK_BF16, ld_out, stride_out, 0.f, 0.f};
  return orthogonal(ctx, s, to, batch, m, n, steps, coef, (cudaStream_t)stream);
}

int rtopk_orthogonal_update(rtopk_matrix* ctx, const float* grad, int64_t ld_g, int64_t stride_g, float* momentum, int64_t ld_v, int64_t stride_v, float* weights,
                            int64_t ld_w, int64_t stride_w, int64_t batch, int64_t m, int64_t n, float eta, float mu, int nesterov, float decay, float scale,
                            int steps, const float* coef, float eps, void* stream) {
  MAT_TRY(check_orth(ctx, batch, m, n, steps, coef, eps));
  if (bad_view(grad, 4, batch, m, n, ld_g, stride_g) || bad_view(momentum, 4, batch, m, n, ld_v, stride_v) || bad_view(weights, 4, batch, m, n, ld_w, stride_w))
    return RTOPK_ERR_INVALID_ARG;
  if (!(eta >= 0.f) || !std::isfinite(eta) || !(mu >= 0.f && mu < 1.f) || !(decay >= 0.f) || !std::isfinite(decay) || !std::isfinite(scale)) return RTOPK_ERR_INVALID_ARG;
  OnDevice on(ctx->device);
  if (!on.ok) return fail(ctx, cudaErrorInvalidDevice);
  Source s = {};
  s.src = grad, s.ld = ld_g, s.stride = stride_g, s.eps = eps;
  s.vec = rows_aligned(grad, 4, batch, ld_g, stride_g, 16), s.v_vec = rows_aligned(momentum, 4, batch, ld_v, stride_v, 16);
  s.v = momentum, s.v_ld = ld_v, s.v_stride = stride_v, s.mu = mu, s.nesterov = nesterov != 0;
  const Target to = {EPI_UPDATE, weights, 0, ld_w, stride_w, (float)(1.0 - (double)eta * (double)decay), (float)((double)eta * (double)scale)};
  return orthogonal(ctx, s, to, batch, m, n, steps, coef, (cudaStream_t)stream);
}

int rtopk_code_weights(rtopk_matrix* ctx, const void* weights, int dtype, int64_t ld_w, int64_t n_out, int64_t n_in, int8_t* codes, int64_t ld_codes, int8_t* codes_t,
                       int64_t ld_t, float* scales, void* stream) {
  MAT_TRY(check_coded(ctx, 0, n_out, n_in));
  if (bad_dtype(dtype) || bad_view(weights, elem(dtype), 1, n_out, n_in, ld_w, 0) || bad_codes(codes, ld_codes, n_in) || (codes_t && bad_codes(codes_t, ld_t, n_out)) ||
      !scales || !aligned_to(scales, 4))
    return RTOPK_ERR_INVALID_ARG;
  if (codes_t && n_out > 128 * kBatchMax) return RTOPK_ERR_UNSUPPORTED;
  OnDevice on(ctx->device);
  if (!on.ok) return fail(ctx, cudaErrorInvalidDevice);
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == RTOPK_F32) MAT_TRY(code_rows(ctx, (const float*)weights, ld_w, n_out, n_in, nullptr, codes, ld_codes, scales, st));
  else MAT_TRY(code_rows(ctx, (const __nv_bfloat16*)weights, ld_w, n_out, n_in, nullptr, codes, ld_codes, scales, st));
  if (codes_t)
    MAT_TRY(launch(ctx, k_codes_transpose, dim3((unsigned)ceil_div(n_in, 64), (unsigned)ceil_div(n_out, 128)), 256, 0, st, codes, ld_codes, n_out, n_in, codes_t, ld_t));
  return RTOPK_OK;
}

int rtopk_coded_scratch(int64_t tokens, int64_t n_out, int64_t n_in, int64_t* bytes) {
  if (!bytes || tokens < 0 || n_out < 1 || n_in < 1 || tokens > kDimMax || n_out > kDimMax || n_in > kDimMax) return RTOPK_ERR_INVALID_ARG;
  Carve c{nullptr};
  CodedScratch w(c, tokens, n_out, n_in);
  *bytes = c.at;
  return RTOPK_OK;
}

int rtopk_coded_product(rtopk_matrix* ctx, const void* x, int dtype, int64_t ld_x, const int8_t* codes, int64_t ld_codes, const float* scales, int64_t tokens,
                        int64_t n_out, int64_t n_in, void* out, int64_t ld_out, void* stream) {
  MAT_TRY(check_coded(ctx, tokens, n_out, n_in));
  if (bad_dtype(dtype) || bad_codes(codes, ld_codes, n_in) || !scales || !aligned_to(scales, 4)) return RTOPK_ERR_INVALID_ARG;
  if (tokens && (bad_view(x, elem(dtype), 1, tokens, n_in, ld_x, 0) || bad_view(out, elem(dtype), 1, tokens, n_out, ld_out, 0))) return RTOPK_ERR_INVALID_ARG;
  if (n_in > kDepthMax) return RTOPK_ERR_UNSUPPORTED;
  if (!tokens) return RTOPK_OK;
  int64_t need = 0;
  rtopk_coded_scratch(tokens, n_out, n_in, &need);
  if (need > ctx->scratch_bytes) return RTOPK_ERR_INVALID_ARG;
  OnDevice on(ctx->device);
  if (!on.ok) return fail(ctx, cudaErrorInvalidDevice);
  if (dtype == RTOPK_F32) return product(ctx, (const float*)x, ld_x, codes, ld_codes, scales, tokens, n_out, n_in, (float*)out, ld_out, (cudaStream_t)stream);
  return product(ctx, (const __nv_bfloat16*)x, ld_x, codes, ld_codes, scales, tokens, n_out, n_in, (__nv_bfloat16*)out, ld_out, (cudaStream_t)stream);
}

int rtopk_coded_gradients(rtopk_matrix* ctx, const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, int dtype, const int8_t* codes_t, int64_t ld_t,
                          const float* scales, int64_t tokens, int64_t n_out, int64_t n_in, void* dx, int64_t ld_dx, void* dw, int dw_dtype, int64_t ld_dw, void* stream) {
  MAT_TRY(check_coded(ctx, tokens, n_out, n_in));
  if (bad_dtype(dtype) || (!dx && !dw) || (tokens && bad_view(dy, elem(dtype), 1, tokens, n_out, ld_dy, 0))) return RTOPK_ERR_INVALID_ARG;
  if (dx && ((tokens && bad_view(dx, elem(dtype), 1, tokens, n_in, ld_dx, 0)) || bad_codes(codes_t, ld_t, n_out) || !scales || !aligned_to(scales, 4)))
    return RTOPK_ERR_INVALID_ARG;
  if (dw && (bad_dtype(dw_dtype) || bad_view(dw, elem(dw_dtype), 1, n_out, n_in, ld_dw, 0) || (tokens && bad_view(x, elem(dtype), 1, tokens, n_in, ld_x, 0))))
    return RTOPK_ERR_INVALID_ARG;
  if ((dx && n_out > kDepthMax) || (dw && tokens > kDepthMax)) return RTOPK_ERR_UNSUPPORTED;
  int64_t need = 0;
  rtopk_coded_scratch(tokens, n_out, n_in, &need);
  if (tokens && need > ctx->scratch_bytes) return RTOPK_ERR_INVALID_ARG;
  OnDevice on(ctx->device);
  if (!on.ok) return fail(ctx, cudaErrorInvalidDevice);
  cudaStream_t st = (cudaStream_t)stream;
  if (!tokens) {      // an empty sum
    if (dw) MAT_CUDA(cudaMemset2DAsync(dw, ld_dw * elem(dw_dtype), 0, n_in * elem(dw_dtype), n_out, st));
    return RTOPK_OK;
  }
  if (dtype == RTOPK_F32)
    return gradients(ctx, (const float*)dy, ld_dy, (const float*)x, ld_x, codes_t, ld_t, scales, tokens, n_out, n_in, (float*)dx, ld_dx, dw, dw_dtype, ld_dw, st);
  return gradients(ctx, (const __nv_bfloat16*)dy, ld_dy, (const __nv_bfloat16*)x, ld_x, codes_t, ld_t, scales, tokens, n_out, n_in, (__nv_bfloat16*)dx, ld_dx, dw, dw_dtype, ld_dw, st);
}

}  // extern "C"
