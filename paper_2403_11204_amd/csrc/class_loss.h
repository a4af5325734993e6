// Internal launch interface of the losses over the classes of a linear layer (class_loss.hip: what is done for each row and entry,
// class_products.hip: the matrix products); the C ABI's host code for them is in losses.hip.  dtype: 0 = float32, 1 = bf16.  Leading dimensions are in
// elements.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace slp {

// C[m][n] = sum over k of A[m][k] B[n][k], both operands of one type, rows on 16-byte boundaries and zero from K up to the next 16 bytes.  What becomes of
// the sums s:
//   PRODUCT_STATS  rows of x against classes: z = (s + bias[n]) times per_t; for each row and span of columns the largest z and sum of exp(z - it)
//   PRODUCT_PROB   the same z: p = exp(z - norm[m].x) norm[m].y to P; if wanted the sums of P's columns over parts of the rows
//   PRODUCT_DX     P W: B lies the other way, as [K][ldb]
//   PRODUCT_DW     P^T x: both do, A as [K][lda], B as [K][ldb]; either: alpha s to a matrix of either type, or s to (or added to) partial sums, one matrix for each
//                  part of the contraction
// An operand that lies the other way has its columns' last 16 bytes to itself, and is smaller than 2 GiB.
//   PRODUCT_Z      partial sums of rows of x against classes, of few tiles with a long contraction
enum { PRODUCT_STATS = 0, PRODUCT_PROB = 1, PRODUCT_DX = 2, PRODUCT_DW = 3, PRODUCT_Z = 4 };
struct ClassProduct {
  const void *a, *b;
  int64_t lda, ldb;
  int M, N, K;
  // STATS and PROB
  const float* bias;        // [N], may be null
  float per_t;
  float2* stats;            // [stats_spans(M, N, K)][M]: (largest, sum)
  float* z;                 // [M][ldz], may be null: z itself of the first zcols columns
  int64_t ldz;
  int zcols;
  const float2* norm;       // [M]: the row's largest z (+infinity: the row does not count, its P is zero), 1 / its sum of exp(z - that)
  const int32_t* labels;    // [M], may be null: class from whose probability 1 is taken
  int label0;               // column 0's class
  void* p;                  // [M][ldp], written up to the next 8 columns
  int64_t ldp;
  float* sums;              // [sum_parts(M, N, K)][N], may be null
  // DX, DW and Z
  void* out;                // [M][ldo] of out_dtype, any alignment
  int64_t ldo;
  int out_dtype;
  const float* alpha;       // device
  float* work;              // not null: partial sums instead, [parts][M][N rounded up to 4]
  int parts;                // of the contraction (1 where work is null)
  bool add;                 // to what work holds
};
// parts of a product's contraction that fill the chip: for PRODUCT_DX and PRODUCT_DW
int class_parts(int dtype, int M, int N, int K);
int z_parts(int dtype, int M, int N, int K);      // 0: PRODUCT_STATS
int stats_spans(int dtype, int M, int N, int K);
// of `classes`, as many as one launch of PRODUCT_STATS or PRODUCT_DW had better take; others: rows and dim, or dim and rows
int whole_rounds(int dtype, int kind, int classes, int others, int K);
int sum_parts(int dtype, int M, int N, int K);
hipError_t launch_class_product(int dtype, int kind, const ClassProduct& g, hipStream_t s);
// dX, and dW with it (`together`) where both are a few small tiles
hipError_t launch_class_gradients(int dtype, const ClassProduct& x, const ClassProduct& w, bool& together, hipStream_t s);

// The rows' targets: class ids (a class id outside [0, classes) is none), and for a distillation the teacher's logits of them.
struct Targets {
  const void* ids;          // [rows][ldids], int32 or int64
  int64_t ldids;
  int ids64;
  const void* top;          // [rows][ldtop] of top_dtype; null: one class for each row, with probability 1
  int64_t ldtop;
  int top_dtype;
  int k;
  float per_t;              // 1 / temperature
};
// zt[row][j] = (x[row] . w[ids[row][j]] + bias) per_t, for classes from `kept` on (the others' logits are kept)
struct TargetLogits {
  const void *x, *w;
  int64_t ldx, ldw;
  const float* bias;
  int rows, classes, dim, kept;
  Targets t;
  float* zt;                // [rows][k]
};
hipError_t launch_target_logits(int dtype, const TargetLogits& a, hipStream_t s);

// From the spans' statistics, or from partial sums of the logits, to each row's log-sum-exp, its loss, what its gradient needs.
struct RowLoss {
  const float2* stats;      // [spans][rows]
  int spans;
  const float* work;        // not null: [parts][rows][classes rounded up to 4], the logits without bias; z, of all classes, is then written from them
  int parts;
  const float* bias;
  int rows, classes;
  Targets t;
  float* z;                 // [rows][ldz]: the logits of classes below `kept`
  int64_t ldz;
  int kept;
  float* zt;                // [rows][k]: of the others; written where kept
  float square_t;           // temperature squared
  float *lse, *losses;      // [rows]
  float2* norm;             // [rows]: see ClassProduct
  float* p;                 // [rows][k], may be null where t.top is: the teacher's probabilities, of all the row's entries of that class
                            // together at the first of them, -1 at the others; 0 where none counts
  int32_t* labels;          // [rows], may be null: the row's class or -1
  unsigned long long* fixed;      // [classes], may be null: cleared on the way
  double2* means;           // [row_groups(this)]: sum of the losses and number of the rows that count, of a group of rows
  float* loss;              // may be null: their mean, where there is one group
};
hipError_t launch_row_loss(const RowLoss& a, hipStream_t s);
int row_groups(const RowLoss& a);
// What follows from all rows: *loss = mean of those that count (0 where none does), *alpha = scale / their number (0); xz = the rows of x, zeros for those that do not
// count and up to the next multiple of 8 columns (may be null; x null: it holds the others already)
struct AllRows {
  const double2* means;     // of `groups` groups of rows
  int groups;
  const float2* norm;
  int rows, dim;
  float scale;
  float *loss, *alpha;
  const void* x;
  int64_t ldx;
  void* xz;
  int64_t ldxz;
};
hipError_t launch_all_rows(int dtype, const AllRows& a, hipStream_t s);

// A distillation's targets: softmax - (the probability of all the row's entries of that class) to P, in classes [first, first + columns)
struct TargetFix {
  Targets t;
  int rows, classes, dtype;
  const float *zt, *p;
  const float2* norm;
  int first, columns;
  void* P;
  int64_t ldp;
  unsigned long long* fixed;      // [columns], may be null: what the targets add to the sums of P's columns, in units of 2^-40 ...
  float* sums;                    // ... and the sums, NaN where that is (may be null)
};
hipError_t launch_target_fix(const TargetFix& a, hipStream_t s);
// P of a piece whose logits are kept, targets and all, and (all may be null) launch_all_rows on the way: rows [rows][ldz] of z from the piece's first class on; sums: as PRODUCT_PROB's, kept_sum_parts(rows) of them
hipError_t launch_kept_prob(const TargetFix& a, const float* z, int64_t ldz, const int32_t* labels, const AllRows* all, hipStream_t s);
int kept_sum_parts(int rows, int columns);
bool fixes_targets(int k, int columns);       // whether it does without `fixed`

// dbias[c] = alpha (sum over the parts of sums[part][c] + fixed[c] 2^-40)
struct BiasGradient {
  const float* sums;        // [parts][columns]
  int parts, columns;
  const unsigned long long* fixed;
  const float* alpha;
  float* dbias;
};

// out[r][c] = in[r][c], zero from cols up to the next multiple of 8
hipError_t launch_pad_rows(int dtype, const void* in, int64_t ldin, int rows, int cols, void* out, int64_t ldo, hipStream_t s);
hipError_t launch_zero(int dtype, void* out, int64_t ldo, int rows, int cols, hipStream_t s);
// out = alpha * sum over the parts, rounded to the type (no rows: nothing of it), and (bias may be null) a bias's gradient on the way
hipError_t launch_join_parts(int dtype, const float* work, int parts, int rows, int cols, const float* alpha, void* out, int64_t ldo, const BiasGradient* bias, hipStream_t s);

}  // namespace slp
