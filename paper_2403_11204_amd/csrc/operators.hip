// C ABI of the 8-bit operators and of gradient clipping (see include/slp.h for the contract).  Host code only: every argument is checked
// before anything is queued.
#include "../../include/slp.h"

#include "eightbit.h"
#include "operator_checks.h"

using namespace slp;

namespace {

constexpr int64_t kMaxRow8 = 1 << 22;      // bytes of an 8-bit row: a tile of 256 rows is addressed with 32-bit offsets
constexpr int kMaxIntegerK = 131071;       // 131071 * 128^2 < 2^31
constexpr int64_t kMaxElements = (int64_t)1 << 34;      // of a matrix: a grid has fewer than 2^32 threads

int check_sides(const char* who, int rows, int cols) {
  if (rows < 0 || cols < 0) return fail(SLP_ERR_ARG, "%s: negative size (%d, %d)", who, rows, cols);
  if (rows > kMaxSide || cols > kMaxSide) return fail(SLP_ERR_SHAPE, "%s: sizes up to %d (got %d, %d)", who, kMaxSide, rows, cols);
  if ((int64_t)rows * cols > kMaxElements) return fail(SLP_ERR_SHAPE, "%s: a matrix of %d x %d", who, rows, cols);
  return SLP_OK;
}

// An 8-bit matrix with rows of `cols` elements.
int check_eight(const char* who, const char* what, const void* q, int64_t ldq, const void* scales, int64_t lds, int cols) {
  if (!q || !scales) return fail(SLP_ERR_ARG, "%s: %s needs values and scales", who, what);
  if (ldq < cols || ldq > kMaxRow8) return fail(SLP_ERR_SHAPE, "%s: leading dimension %lld of %s, rows of %d, at most %lld", who, (long long)ldq, what, cols, (long long)kMaxRow8);
  if (lds < (cols + kScaleBlock - 1) / kScaleBlock || lds > kMaxRow8)
    return fail(SLP_ERR_SHAPE, "%s: leading dimension %lld of the scales of %s, rows of %d", who, (long long)lds, what, cols);
  if (off(q, 16) || ldq % 16) return fail(SLP_ERR_ALLOC, "%s: rows of %s must start on 16-byte boundaries", who, what);
  if (off(scales, 4) || lds % 4) return fail(SLP_ERR_ALLOC, "%s: rows of the scales of %s must start on 4-byte boundaries", who, what);
  return SLP_OK;
}

// A matrix of integers with rows of `cols` elements and a scale each.
int check_integers(const char* who, const char* what, const void* q, int64_t ldq, const float* scales, int cols) {
  if (ldq < cols || ldq > kMaxRow8) return fail(SLP_ERR_SHAPE, "%s: leading dimension %lld of %s, rows of %d, at most %lld", who, (long long)ldq, what, cols, (long long)kMaxRow8);
  if (off(q, 16) || ldq % 16) return fail(SLP_ERR_ALLOC, "%s: rows of %s must start on 16-byte boundaries", who, what);
  if (off(scales, 4)) return fail(SLP_ERR_ALLOC, "%s: the scales of %s are not on an element's boundary", who, what);
  return SLP_OK;
}

int chunk_groups(int64_t chunks) { return (int)(chunks < 1 ? 1 : chunks < kClipMaxGroups ? chunks : kClipMaxGroups); }
int64_t chunks_of(int64_t count, int dt) { return (count * (int64_t)size_of(dt) + kClipChunk - 1) / kClipChunk; }

// Partial sums of all launches; -1 where a tensor has more chunks than fit.
int clip_partials(const int64_t* counts, const int* dts, int n) {
  int64_t all = 0;
  for (int i = 0; i < n; i += kClipTensors) {
    int64_t chunks = 0;
    for (int k = i; k < n && k < i + kClipTensors; ++k) {
      if (counts[k] < 0 || counts[k] > ((int64_t)1 << 43)) return -1;
      chunks += chunks_of(counts[k], dts[k]);
      if (chunks > INT32_MAX) return -1;
    }
    all += chunk_groups(chunks);
    if (all > INT32_MAX / 8) return -1;
  }
  return (int)all;
}

int clip_run(const char* who, const void* const* in, void* const* out, const int64_t* counts, const int* dts, int n, bool scale, float max_norm,
             float* norm_out, void* workspace, size_t workspace_bytes, hipStream_t s) {
  if (n < 0) return fail(SLP_ERR_ARG, "%s: negative number of tensors", who);
  if (n && (!in || !counts || !dts)) return fail(SLP_ERR_ARG, "%s: null array", who);
  for (int i = 0; i < n; ++i) {
    if (!known(dts[i])) return fail(SLP_ERR_ARG, "%s: unknown dtype %d of tensor %d", who, dts[i], i);
    if (counts[i] < 0) return fail(SLP_ERR_ARG, "%s: negative size of tensor %d", who, i);
    if (counts[i] && (!in[i] || (scale && out && !out[i]))) return fail(SLP_ERR_ARG, "%s: tensor %d is null", who, i);
    if (counts[i] && (off(in[i], size_of(dts[i])) || (scale && out && off(out[i], size_of(dts[i])))))
      return fail(SLP_ERR_ALLOC, "%s: tensor %d is not on an element's boundary", who, i);
  }
  const int partials = clip_partials(counts, dts, n);
  if (partials < 0) return fail(SLP_ERR_SHAPE, "%s: too many elements", who);
  SLP_CHECK(check_work(who, workspace, workspace_bytes, slp_gradient_norm_workspace_bytes(n)));
  double* const sums = (double*)workspace;
  for (int pass = 0; pass < (scale ? 2 : 1); ++pass) {
    int done = 0;
    for (int i = 0; i < n || (i == 0 && n == 0); i += kClipTensors) {
      ClipTable t{};
      for (int k = i; k < n && k < i + kClipTensors; ++k) {
        t.in[t.n] = in[k];
        t.out[t.n] = out ? out[k] : const_cast<void*>(in[k]);
        t.count[t.n] = counts[k];
        t.bf16 |= (uint64_t)(dts[k] == SLP_BF16) << t.n;
        t.chunk0[t.n + 1] = t.chunk0[t.n] + (int)chunks_of(counts[k], dts[k]);
        ++t.n;
      }
      const int groups = chunk_groups(t.chunk0[t.n]);
      if (pass == 0) HIP_TRY(launch_square_sums(t, groups, sums + done, s));
      else HIP_TRY(launch_scale(t, groups, sums, partials, max_norm, i == 0 ? norm_out : nullptr, s));
      done += groups;
    }
  }
  if (!scale) HIP_TRY(launch_norm_of(sums, partials, norm_out, s));
  return SLP_OK;
}

}  // namespace

extern "C" {

size_t slp_quantize_workspace_bytes(int rows, int cols) {
  return rows > 0 && cols > 0 && rows <= kMaxSide && cols <= kMaxSide ? quantize_floats(rows, cols) * sizeof(float) : 0;
}

int slp_quantize(const void* x, int64_t ldx, const void* mask, int64_t ldmask, int dt, int rows, int cols, int block, void* q, int64_t ldq,
                 void* scales, int64_t lds, void* qt, int64_t ldqt, void* scales_t, int64_t ldst, float* column_sums, void* workspace,
                 size_t workspace_bytes, slp_stream stream) {
  const char* const who = "slp_quantize";
  if (!known(dt)) return fail(SLP_ERR_ARG, "%s: unknown dtype %d", who, dt);
  if (block != 1 && block != kScaleBlock) return fail(SLP_ERR_ARG, "%s: blocks of 1 or %d rows (got %d)", who, kScaleBlock, block);
  SLP_CHECK(check_sides(who, rows, cols));
  if (off(column_sums, 4)) return fail(SLP_ERR_ALLOC, "%s: the sums are not on an element's boundary", who);
  if (rows == 0 && cols > 0 && column_sums) {       // sums of nothing
    HIP_TRY(launch_sum_rows(nullptr, 0, cols, column_sums, (hipStream_t)stream));
    return SLP_OK;
  }
  if (rows == 0 || cols == 0) return SLP_OK;
  if (!q && !scales && !qt && !scales_t) return fail(SLP_ERR_ARG, "%s: no output", who);
  if (q || scales) SLP_CHECK(check_eight(who, "the row-major output", q, ldq, scales, lds, cols));
  if (qt || scales_t) SLP_CHECK(check_eight(who, "the transposed output", qt, ldqt, scales_t, ldst, rows));
  if (!x) return fail(SLP_ERR_ARG, "%s: null pointer", who);
  SLP_CHECK(check_dense(who, "x", x, ldx, cols, dt));
  if (mask) SLP_CHECK(check_dense(who, "mask", mask, ldmask, cols, dt));
  if (column_sums) SLP_CHECK(check_work(who, workspace, workspace_bytes, slp_quantize_workspace_bytes(rows, cols)));
  const QuantizeArgs a{x, mask, (uint8_t*)q, (uint8_t*)scales, (uint8_t*)qt, (uint8_t*)scales_t, column_sums, (float*)workspace, ldx, ldmask, ldq, lds,
                       ldqt, ldst, rows, cols, block};
  HIP_TRY(launch_quantize(dt, a, (hipStream_t)stream));
  return SLP_OK;
}

size_t slp_product_workspace_bytes(int M, int N, int K) {
  return M > 0 && N > 0 && K >= 0 && M <= kMaxSide && N <= kMaxSide && K <= kMaxSide ? product_floats(M, N, K) * sizeof(float) : 0;
}

int slp_product(const void* a, int64_t lda, const void* a_scales, int64_t ldsa, int a_block, const void* b, int64_t ldb, const void* b_scales,
                int64_t ldsb, int b_block, const float* bias, int relu, int M, int N, int K, void* out, int64_t ldo, int dt, void* workspace,
                size_t workspace_bytes, slp_stream stream) {
  const char* const who = "slp_product";
  const bool exact = dt >= 0 && (dt & SLP_FLOAT32_SUMS) != 0;
  if (exact) dt &= ~SLP_FLOAT32_SUMS;
  if (!known(dt)) return fail(SLP_ERR_ARG, "%s: unknown dtype %d", who, dt);
  if ((a_block != 1 && a_block != kScaleBlock) || (b_block != 1 && b_block != kScaleBlock))
    return fail(SLP_ERR_ARG, "%s: blocks of 1 or %d rows (got %d, %d)", who, kScaleBlock, a_block, b_block);
  SLP_CHECK(check_sides(who, M, N));
  SLP_CHECK(check_sides(who, K, 1));
  if (M == 0 || N == 0) return SLP_OK;
  if (!out) return fail(SLP_ERR_ARG, "%s: null pointer", who);
  SLP_CHECK(check_dense(who, "out", out, ldo, N, dt));
  if (K > 0) {
    SLP_CHECK(check_eight(who, "a", a, lda, a_scales, ldsa, K));
    SLP_CHECK(check_eight(who, "b", b, ldb, b_scales, ldsb, K));
  } else {
    lda = ldsa = ldb = ldsb = 0;       // unchecked, and the kernels' bounds are made of them
  }
  if (bias && off(bias, 4)) return fail(SLP_ERR_ALLOC, "%s: bias is not on an element's boundary", who);
  SLP_CHECK(check_work(who, workspace, workspace_bytes, slp_product_workspace_bytes(M, N, K)));
  const ProductArgs g{(const uint8_t*)a, (const uint8_t*)a_scales, (const uint8_t*)b, (const uint8_t*)b_scales, lda, ldsa, ldb, ldsb,
                      a_block == 1 ? 0 : 7, b_block == 1 ? 0 : 7, M, N, K, bias, relu, out, ldo, dt, exact, (float*)workspace};
  HIP_TRY(launch_product(g, (hipStream_t)stream));
  return SLP_OK;
}

int slp_quantize_integers(const void* x, int64_t ldx, int dt, int rows, int cols, void* q, int64_t ldq, float* scales, slp_stream stream) {
  const char* const who = "slp_quantize_integers";
  if (!known(dt)) return fail(SLP_ERR_ARG, "%s: unknown dtype %d", who, dt);
  SLP_CHECK(check_sides(who, rows, cols));
  if (rows == 0) return SLP_OK;
  if (!scales || (cols > 0 && (!x || !q))) return fail(SLP_ERR_ARG, "%s: null pointer", who);
  SLP_CHECK(check_integers(who, "q", q, ldq, scales, cols));
  SLP_CHECK(check_dense(who, "x", x, ldx, cols, dt));
  const IntegersArgs a{x, (int8_t*)q, scales, ldx, ldq, rows, cols};
  HIP_TRY(launch_quantize_integers(dt, a, (hipStream_t)stream));
  return SLP_OK;
}

size_t slp_product_integers_workspace_bytes(int M, int N, int K) {
  return M > 0 && N > 0 && K >= 0 && M <= kMaxSide && N <= kMaxSide && K <= kMaxIntegerK ? integer_product_words(M, N, K) * sizeof(int32_t) : 0;
}

int slp_product_integers(const void* a, int64_t lda, const float* a_scales, const void* b, int64_t ldb, const float* b_scales, const float* bias, int relu, int M, int N, int K,
                         void* out, int64_t ldo, int dt, void* workspace, size_t workspace_bytes, slp_stream stream) {
  const char* const who = "slp_product_integers";
  if (!known(dt)) return fail(SLP_ERR_ARG, "%s: unknown dtype %d", who, dt);
  SLP_CHECK(check_sides(who, M, N));
  if (K < 0) return fail(SLP_ERR_ARG, "%s: negative size %d", who, K);
  if (K > kMaxIntegerK) return fail(SLP_ERR_SHAPE, "%s: contractions of up to %d, whose sums fit 32 bits (got %d)", who, kMaxIntegerK, K);
  if (M == 0 || N == 0) return SLP_OK;
  if (!out || !a_scales || !b_scales || (K > 0 && (!a || !b))) return fail(SLP_ERR_ARG, "%s: null pointer", who);
  SLP_CHECK(check_dense(who, "out", out, ldo, N, dt));
  if (K == 0) lda = ldb = 0;             // (the kernels' bounds are made of them)
  SLP_CHECK(check_integers(who, "a", a, lda, a_scales, K));
  SLP_CHECK(check_integers(who, "b", b, ldb, b_scales, K));
  if (off(bias, 4)) return fail(SLP_ERR_ALLOC, "%s: bias is not on an element's boundary", who);
  SLP_CHECK(check_work(who, workspace, workspace_bytes, slp_product_integers_workspace_bytes(M, N, K)));
  const IntegerProductArgs g{(const int8_t*)a, (const int8_t*)b, a_scales, b_scales, lda, ldb, M, N, K, bias, relu, out, ldo, dt, (int32_t*)workspace};
  HIP_TRY(launch_integer_product(g, (hipStream_t)stream));
  return SLP_OK;
}

int slp_rmsnorm(const void* x, int64_t ldx, const void* residual, int64_t ldr, const float* gamma, float eps, int dt, int rows, int dim, void* h,
                int64_t ldh, void* y, int64_t ldy, void* q, int64_t ldq, void* scales, int64_t lds, float* rstd, slp_stream stream) {
  const char* const who = "slp_rmsnorm";
  if (!known(dt)) return fail(SLP_ERR_ARG, "%s: unknown dtype %d", who, dt);
  if (!(eps >= 0.0f)) return fail(SLP_ERR_ARG, "%s: eps must not be negative", who);
  SLP_CHECK(check_sides(who, rows, dim));
  if (dim == 0) return fail(SLP_ERR_ARG, "%s: rows of no elements have no mean", who);
  if (q || scales) SLP_CHECK(check_eight(who, "the 8-bit output", q, ldq, scales, lds, dim));
  if (rows == 0) return SLP_OK;
  if (!x) return fail(SLP_ERR_ARG, "%s: null pointer", who);
  if (residual && !h) return fail(SLP_ERR_ARG, "%s: a residual needs h for the sum", who);
  SLP_CHECK(check_dense(who, "x", x, ldx, dim, dt));
  if (residual) SLP_CHECK(check_dense(who, "residual", residual, ldr, dim, dt));
  if (h) SLP_CHECK(check_dense(who, "h", h, ldh, dim, dt));
  if (y) SLP_CHECK(check_dense(who, "y", y, ldy, dim, dt));
  if (off(gamma, 4) || off(rstd, 4)) return fail(SLP_ERR_ALLOC, "%s: gamma or rstd is not on an element's boundary", who);
  const NormArgs a{x, residual, gamma, h, y, (uint8_t*)q, (uint8_t*)scales, rstd, ldx, ldr, ldh, ldy, ldq, lds, rows, dim, eps};
  HIP_TRY(launch_rmsnorm(dt, a, (hipStream_t)stream));
  return SLP_OK;
}

size_t slp_rmsnorm_backward_workspace_bytes(int rows, int dim) {
  return rows > 0 && dim > 0 && rows <= kMaxSide && dim <= kMaxSide ? rmsnorm_backward_floats(rows, dim) * sizeof(float) : 0;
}

int slp_rmsnorm_backward(const void* dy, int64_t lddy, const void* h, int64_t ldh, const float* gamma, const float* rstd, const void* dh, int64_t lddh,
                         int dt, int rows, int dim, void* dx, int64_t lddx, float* dgamma, void* workspace, size_t workspace_bytes, slp_stream stream) {
  const char* const who = "slp_rmsnorm_backward";
  if (!known(dt)) return fail(SLP_ERR_ARG, "%s: unknown dtype %d", who, dt);
  SLP_CHECK(check_sides(who, rows, dim));
  if (dim == 0) return fail(SLP_ERR_ARG, "%s: rows of no elements have no mean", who);
  if (off(dgamma, 4) || off(gamma, 4) || off(rstd, 4)) return fail(SLP_ERR_ALLOC, "%s: gamma, dgamma or rstd is not on an element's boundary", who);
  if (rows == 0) {
    if (dgamma) HIP_TRY(launch_sum_rows(nullptr, 0, dim, dgamma, (hipStream_t)stream));
    return SLP_OK;
  }
  if (!dy || !h || !rstd || !dx) return fail(SLP_ERR_ARG, "%s: null pointer", who);
  SLP_CHECK(check_dense(who, "dy", dy, lddy, dim, dt));
  SLP_CHECK(check_dense(who, "h", h, ldh, dim, dt));
  SLP_CHECK(check_dense(who, "dx", dx, lddx, dim, dt));
  if (dh) SLP_CHECK(check_dense(who, "dh", dh, lddh, dim, dt));
  SLP_CHECK(check_work(who, workspace, workspace_bytes, slp_rmsnorm_backward_workspace_bytes(rows, dim)));
  const NormBackArgs a{dy, h, dh, gamma, rstd, dx, dgamma, lddy, ldh, lddh, lddx, rows, dim, (float*)workspace};
  HIP_TRY(launch_rmsnorm_backward(dt, a, (hipStream_t)stream));
  return SLP_OK;
}

size_t slp_gradient_norm_workspace_bytes(int n) {
  return n < 0 ? 0 : (size_t)(n / kClipTensors + 1) * kClipMaxGroups * sizeof(double);
}

int slp_gradient_norm(const void* const* tensors, const int64_t* counts, const int* dts, int n, float* norm_out, void* workspace,
                      size_t workspace_bytes, slp_stream stream) {
  if (!norm_out) return fail(SLP_ERR_ARG, "slp_gradient_norm: null pointer");
  return clip_run("slp_gradient_norm", tensors, nullptr, counts, dts, n, false, 0.0f, norm_out, workspace, workspace_bytes, (hipStream_t)stream);
}

int slp_clip_gradients(const void* const* tensors, void* const* out, const int64_t* counts, const int* dts, int n, float max_norm, float* norm_out,
                       void* workspace, size_t workspace_bytes, slp_stream stream) {
  if (!(max_norm > 0.0f)) return fail(SLP_ERR_ARG, "slp_clip_gradients: max_norm must be positive");
  return clip_run("slp_clip_gradients", tensors, out, counts, dts, n, true, max_norm, norm_out, workspace, workspace_bytes, (hipStream_t)stream);
}

}  // extern "C"
