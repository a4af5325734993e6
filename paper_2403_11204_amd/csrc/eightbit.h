// Internal launch interface of the 8-bit operators (norm.hip, quantize.hip, product.hip) and of gradient clipping (clip.hip); the C ABI's
// host code for them is in operators.hip.  dtype: 0 = float32, 1 = bf16.  Leading dimensions are in elements.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace slp {

constexpr int kScaleBlock = 128;      // elements of a row that share a scale

struct NormArgs {
  const void *x, *r;        // [rows][dim]; r may be null
  const float* gamma;       // [dim], may be null: ones
  void* h;                  // x + r, rounded to the type; null only where r is
  void* y;                  // the norm in the type, may be null
  uint8_t *q, *scales;      // the norm in 8 bits, may be null
  float* rstd;              // may be null
  int64_t ldx, ldr, ldh, ldy, ldq, lds;
  int rows, dim;
  float eps;
};
hipError_t launch_rmsnorm(int dtype, const NormArgs& a, hipStream_t s);

struct NormBackArgs {
  const void *dy, *h, *dh;  // dh may be null
  const float *gamma, *rstd;
  void* dx;
  float* dgamma;            // may be null
  int64_t lddy, ldh, lddh, lddx;
  int rows, dim;
  float* work;              // rmsnorm_backward_floats(rows, dim)
};
size_t rmsnorm_backward_floats(int rows, int dim);
hipError_t launch_rmsnorm_backward(int dtype, const NormBackArgs& a, hipStream_t s);

struct QuantizeArgs {
  const void *x, *mask;     // [rows][cols]; mask may be null
  uint8_t *q, *scales;      // row-major, may be null
  uint8_t *qt, *scales_t;   // transposed, may be null
  float* sums;              // of the columns, may be null
  float* work;              // quantize_floats(rows, cols), where sums is given
  int64_t ldx, ldmask, ldq, lds, ldqt, ldst;
  int rows, cols;
  int block;                // 1 or 128 rows share a scale
};
size_t quantize_floats(int rows, int cols);
hipError_t launch_quantize(int dtype, const QuantizeArgs& a, hipStream_t s);

// out[c] = sum over i < n of in[i][c], in order of i within a few strands that are then added in order
hipError_t launch_sum_rows(const float* in, int n, int cols, float* out, hipStream_t s);

struct ProductArgs {
  const uint8_t *a, *sa, *b, *sb;
  int64_t lda, ldsa, ldb, ldsb;
  int shift_a, shift_b;     // row of a scale = row of the matrix >> shift (0 or 7)
  int M, N, K;
  const float* bias;        // [N], may be null
  int relu;
  void* out;                // [M][ldo]
  int64_t ldo;
  int out_dtype;
  bool exact;               // float32 sums for a bf16 output, too
  float* work;              // product_floats(M, N, K)
};
size_t product_floats(int M, int N, int K);
hipError_t launch_product(const ProductArgs& a, hipStream_t s);

// Integers: rows of x to q = round(127 x / max|x|), ties to even, and scale = max|x| / 127.
struct IntegersArgs {
  const void* x;
  int8_t* q;
  float* scales;            // [rows]
  int64_t ldx, ldq;
  int rows, cols;
};
hipError_t launch_quantize_integers(int dtype, const IntegersArgs& a, hipStream_t s);
struct IntegerProductArgs {
  const int8_t *a, *b;
  const float *sa, *sb;     // of the rows
  int64_t lda, ldb;
  int M, N, K;
  const float* bias;        // [N], may be null
  int relu;
  void* out;                // [M][ldo]
  int64_t ldo;
  int out_dtype;
  int32_t* work;            // integer_product_words(M, N, K)
};
size_t integer_product_words(int M, int N, int K);
hipError_t launch_integer_product(const IntegerProductArgs& g, hipStream_t s);

constexpr int kClipTensors = 48;      // a launch takes (kernel arguments)
struct ClipTable {
  const void* in[kClipTensors];
  void* out[kClipTensors];
  int64_t count[kClipTensors];
  int chunk0[kClipTensors + 1];       // first chunk of each tensor among the launch's
  uint64_t bf16;                      // bit i: tensor i holds bf16
  int n;
};
constexpr int kClipChunk = 32768;     // bytes
constexpr int kClipMaxGroups = 256;   // workgroups of one launch at most
// partials[0 .. groups) = sums of squares, one a workgroup
hipError_t launch_square_sums(const ClipTable& t, int groups, double* partials, hipStream_t s);
// *norm = sqrt(sum of partials)
hipError_t launch_norm_of(const double* partials, int n, float* norm, hipStream_t s);
// out = c * in with c from the sum of all partials; the first workgroup writes *norm where it is not null
hipError_t launch_scale(const ClipTable& t, int groups, const double* partials, int n, float max_norm, float* norm, hipStream_t s);

}  // namespace slp
