// Losses over the classes of a linear layer: what is done for each row and for each of its targets, around the products in class_products.hip.
//
// With z = x W^T + b, temperature T and a row's targets c(j) of probability p_j (one of probability 1, or a teacher's softmax(top / T)):
//   lse = log sum_v exp(z_v / T)        loss = T^2 sum_j p_j (log p_j + lse - z_c(j) / T)        dz_v = T (exp(z_v / T - lse) - sum of p_j with c(j) = v)
// The logits of the targets are computed apart, in float32: P, which leaves the products rounded to the operands' type, gets exp(z_c / T - lse) - p_j written over
// it, so that nothing cancels among rounded values.
#include "class_loss.h"
#include "eightbit_device.h"

#include <type_traits>

namespace slp {
namespace {

// The class of entry j of a row; -1 where it is none.
__device__ __forceinline__ int class_of(const Targets& t, int64_t row, int j, int classes) {
  if (t.ids64) {
    const int64_t c = ((const int64_t*)t.ids)[row * t.ldids + j];
    return c >= 0 && c < classes ? (int)c : -1;
  }
  const int32_t c = ((const int32_t*)t.ids)[row * t.ldids + j];
  return c >= 0 && c < classes ? c : -1;
}
// The teacher's logit over the temperature; -infinity for an entry that does not count.
__device__ __forceinline__ float teacher(const Targets& t, int64_t row, int j, int classes) {
  const int64_t at = row * t.ldtop + j;
  const float z = (t.top_dtype == 1 ? (float)((const bf16*)t.top)[at] : ((const float*)t.top)[at]) * t.per_t;
  return class_of(t, row, j, classes) < 0 ? -INFINITY : z;
}

// The dot product of a row of x and the row of W that is its class, one wavefront for each target; a workgroup where they are few and each waits for its own loads (1 target of
// 4096 bf16 8.2 us on a wavefront, 5 on a workgroup), 16 lanes where rows are short (6146 x 25 targets of 170 46 / 18).  Many are bound by reading those rows of W: 4096 x 64 targets of 4096 bf16 are 2.1 GB.
template <typename T, int TEAM>
__global__ __launch_bounds__(256) void target_logits_kernel(const TargetLogits a) {
  const int64_t at = (int64_t)blockIdx.x * (256 / TEAM) + threadIdx.x / TEAM;
  const int lane = threadIdx.x % TEAM;
  if (at >= (int64_t)a.rows * a.t.k) return;
  const int64_t row = at / a.t.k;
  const int c = class_of(a.t, row, (int)(at % a.t.k), a.classes);
  if (c < a.kept) return;                // (none, or kept)
  const T* const x = (const T*)a.x + row * a.ldx;
  const T* const w = (const T*)a.w + (int64_t)c * a.ldw;
  float sum = 0.0f;
  for (int d = lane * 8; d < a.dim; d += TEAM * 8) {
    float u[8], v[8];
    load8(x + d, a.dim - d, u);
    load8(w + d, a.dim - d, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += u[e] * v[e];
  }
  sum = TEAM == 16 ? sum_of_16(sum) : sum_of_64(sum);
  if constexpr (TEAM == 256) {
    __shared__ float part[4];
    if ((lane & 63) == 0) part[lane >> 6] = sum;
    __syncthreads();
    sum = (part[0] + part[1]) + (part[2] + part[3]);
  }
  if (lane == 0) a.zt[at] = (sum + (a.bias ? a.bias[c] : 0.0f)) * a.t.per_t;
}

// (largest, sum of exp(z - largest)) of two sets together; the largest of nothing is -infinity
__device__ __forceinline__ float2 joined(float2 a, float2 b) {
  const float most = fmaxf(a.x, b.x);
  return float2{most, (a.x == most ? a.y : a.y * expf(a.x - most)) + (b.x == most ? b.y : b.y * expf(b.x - most))};
}

// Over the lanes of a wavefront.
__device__ __forceinline__ float fmax_of_64(float x) {
  auto step = [&](auto ctrl) { x = fmaxf(x, __builtin_bit_cast(float, dpp<decltype(ctrl)::value>(__builtin_bit_cast(uint32_t, x)))); };
  step(std::integral_constant<int, kSwap1>{});
  step(std::integral_constant<int, kSwap2>{});
  step(std::integral_constant<int, kHalfMirror>{});
  step(std::integral_constant<int, kMirror>{});
  uint32_t u = __builtin_bit_cast(uint32_t, x);
  u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(u, u, false, false));
  uint32_t a = r[0], b = r[1];
  u = __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
  r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(u, u, false, false));
  a = r[0];
  b = r[1];
  return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

// TEAM threads a row: 16; a wavefront where there are few rows; all 256 of a workgroup where there are many spans as well (1 x 131072 classes, 1024 spans: 35 us on 16 threads,
// 5 on 256; 64 x 1000 with 8 entries 8 on 256).  Workgroups behind the rows' clear `fixed`.
template <int TEAM>
__global__ __launch_bounds__(256) void row_loss_kernel(const RowLoss a) {
  constexpr int ROWS = 256 / TEAM;
  __shared__ float2 part[TEAM == 64 ? 1 : 16][TEAM == 16 ? 16 : 1];
  extern __shared__ float2 entries[];          // of a distillation: class and probability of each row's entries
  const int t = threadIdx.x, r = TEAM == 16 ? t % 16 : t / TEAM, s = TEAM == 16 ? t / 16 : t % TEAM, groups = (a.rows + ROWS - 1) / ROWS;
  if ((int)blockIdx.x >= groups) {
    const int64_t i = ((int64_t)(blockIdx.x - groups) * 256 + t) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (i + e < a.classes) a.fixed[i + e] = 0;
    return;
  }
  const int64_t row = (int64_t)blockIdx.x * ROWS + r;
  const bool in = row < a.rows;
  // of the row's threads, in the same order every time
  auto all = [&](float2 mine) {
    if constexpr (TEAM > 16) {
      const float most = fmax_of_64(mine.x);
      mine = float2{most, sum_of_64(mine.x == most ? mine.y : mine.y * expf(mine.x - most))};
    }
    if constexpr (TEAM != 64) {
      constexpr int N = TEAM == 16 ? 16 : 4;
      const int c = TEAM == 16 ? r : 0, at = TEAM == 16 ? s : s >> 6;
      __syncthreads();
      part[at][c] = mine;
      __syncthreads();
      mine = part[0][c];
#pragma unroll
      for (int i = 1; i < N; ++i) mine = joined(mine, part[i][c]);
    }
    return mine;
  };
  auto total = [&](float mine) {
    if constexpr (TEAM > 16) mine = sum_of_64(mine);
    if constexpr (TEAM != 64) {
      constexpr int N = TEAM == 16 ? 16 : 4;
      const int c = TEAM == 16 ? r : 0, at = TEAM == 16 ? s : s >> 6;
      __syncthreads();
      part[at][c].x = mine;
      __syncthreads();
      mine = part[0][c].x;
#pragma unroll
      for (int i = 1; i < N; ++i) mine += part[i][c].x;
    }
    return mine;
  };
  float2 mine = {-INFINITY, 0.0f};
  if (a.work) {
    // four classes at a time; then once more, from what this thread has written itself
    const int64_t ldw = (a.classes + 3) & ~3;
    const float* const work = a.work + row * ldw;
    float* const z = a.z + row * a.ldz;
    if (in)
      for (int c = 4 * s; c < a.classes; c += 4 * TEAM) {
        f32x4 v = *(const f32x4*)(work + c);
#pragma unroll 8
        for (int p = 1; p < a.parts; ++p) v += *(const f32x4*)(work + p * a.rows * ldw + c);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = c + e < a.classes ? (v[e] + (a.bias ? a.bias[c + e] : 0.0f)) * a.t.per_t : -INFINITY;
          mine.x = fmaxf(mine.x, v[e]);
        }
        *(f32x4*)(z + c) = v;
      }
    const float most = all(mine).x, from = most == -INFINITY ? 0.0f : most;
    mine.x = most;
    if (in)
      for (int c = 4 * s; c < a.classes; c += 4 * TEAM) {
        const f32x4 v = *(const f32x4*)(z + c);
#pragma unroll
        for (int e = 0; e < 4; ++e) mine.y += expf(v[e] - from);
      }
  } else if (in) {
    int i = s;
    for (; i + 3 * TEAM < a.spans; i += 4 * TEAM) {        // four loads under way
      float2 v[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = a.stats[(int64_t)(i + q * TEAM) * a.rows + row];
      mine = joined(mine, joined(joined(v[0], v[1]), joined(v[2], v[3])));
    }
    for (; i < a.spans; i += TEAM) mine = joined(mine, a.stats[(int64_t)i * a.rows + row]);
  }
  mine = all(mine);
  const float log_all = logf(mine.y), lse = mine.x + log_all;         // (apart where the logits are so large that their sum is the largest)
  auto logit = [&](int j, int c) {       // of the row's entry j, class c
    const int64_t at = row * a.t.k + j;
    if (c >= a.kept) return a.zt[at];
    const float z = a.z[row * a.ldz + c];
    a.zt[at] = z;
    return z;
  };
  float loss = 0.0f;
  bool counts = false;
  if (!a.t.top) {
    const int c = in ? class_of(a.t, row, 0, a.classes) : -1;
    counts = c >= 0;
    if (counts && s == 0) loss = log_all + (mine.x - logit(0, c));
    if (in && s == 0 && a.labels) a.labels[row] = c;
  } else {
    const int k = in ? a.t.k : 0;
    float2 top = {-INFINITY, 0.0f};
#pragma unroll 4
    for (int j = s; j < k; j += TEAM) {
      const float t = teacher(a.t, row, j, a.classes);
      entries[r * (k | 1) + j] = float2{__builtin_bit_cast(float, class_of(a.t, row, j, a.classes)), t};      // (read again by this thread alone)
      if (t != -INFINITY) top = joined(top, float2{t, 1.0f});
    }
    top = all(top);
    counts = top.y != 0.0f;               // (a NaN counts)
    const float log_sum = logf(top.y);
    for (int j = s; j < k; j += TEAM) {
      const float2 e = entries[r * (k | 1) + j];
      const int c = __builtin_bit_cast(int, e.x);
      const float t = e.y, z = c >= 0 ? logit(j, c) : 0.0f;
      const float logp = t - top.x - log_sum, p = counts && t != -INFINITY ? expf(t - top.x) / top.y : 0.0f;
      entries[r * (k | 1) + j] = float2{__builtin_bit_cast(float, c), p};
      if (p != 0.0f) loss += p * (logp + log_all + (mine.x - z));
    }
    loss = total(loss) * a.square_t;
    // what the entries of one class add up to, at the first of them
    __syncthreads();
    for (int j = s; j < k; j += TEAM) {
      const int c = __builtin_bit_cast(int, entries[r * (k | 1) + j].x);
      float sum = 0.0f;
      bool first = true;
      int i = 0;
      for (; i + 8 <= k; i += 8) {       // eight reads under way
        float2 e[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) e[q] = entries[r * (k | 1) + i + q];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const bool same = __builtin_bit_cast(int, e[q].x) == c;
          sum += same ? e[q].y : 0.0f;
          first &= !same || i + q >= j;
        }
      }
      for (; i < k; ++i) {
        const float2 e = entries[r * (k | 1) + i];
        const bool same = __builtin_bit_cast(int, e.x) == c;
        sum += same ? e.y : 0.0f;
        first &= !same || i >= j;
      }
      a.p[row * k + j] = first ? sum : -1.0f;
    }
  }
  if (in && s == 0) {
    a.lse[row] = lse;
    a.losses[row] = counts ? loss : 0.0f;
    a.norm[row] = float2{!counts ? INFINITY : mine.x == INFINITY ? NAN : mine.x, 1.0f / mine.y};
  }
  // of this workgroup's rows, in their order
  __shared__ double2 group[ROWS];
  if (s == 0) group[r] = in && counts ? double2{(double)loss, 1.0} : double2{0.0, 0.0};
  __syncthreads();
  if (t > 0) return;
  double2 sum = group[0];
#pragma unroll
  for (int i = 1; i < ROWS; ++i) {
    sum.x += group[i].x;
    sum.y += group[i].y;
  }
  a.means[blockIdx.x] = sum;
  if (a.loss) *a.loss = sum.y > 0.0 ? (float)(sum.x / sum.y) : 0.0f;
}

// Block 0: the mean.  The others: 2048 elements each of xz's rows.
template <typename T>
__device__ __forceinline__ void all_rows_block(const AllRows& a, int block) {
  const int t = threadIdx.x;
  if (block == 0) {
    __shared__ double2 sums[4];
    double2 sum = {0.0, 0.0};
#pragma unroll 4
    for (int i = t; i < a.groups; i += 256) {
      const double2 m = a.means[i];
      sum.x += m.x;
      sum.y += m.y;
    }
    for (int step = 32; step > 0; step >>= 1) {
      sum.x += __shfl_xor(sum.x, step);
      sum.y += __shfl_xor(sum.y, step);
    }
    if ((t & 63) == 0) sums[t >> 6] = sum;
    __syncthreads();
    if (t == 0) {
      const double n = (sums[0].y + sums[1].y) + (sums[2].y + sums[3].y);
      *a.loss = n > 0.0 ? (float)(((sums[0].x + sums[1].x) + (sums[2].x + sums[3].x)) / n) : 0.0f;
      *a.alpha = n > 0.0 ? a.scale / (float)n : 0.0f;
    }
    return;
  }
  const int eights = (a.dim + 7) / 8;
  const int64_t at = (int64_t)(block - 1) * 256 + t, row = at / eights;
  const int c = (int)(at % eights) * 8;
  if (row >= a.rows || (!a.x && a.norm[row].x != INFINITY)) return;
  float v[8];
  load8((const T*)a.x + row * a.ldx + c, a.norm[row].x == INFINITY ? 0 : a.dim - c, v);
  store8((T*)a.xz + row * a.ldxz + c, 8, v);
}
template <typename T>
__global__ __launch_bounds__(256) void all_rows_kernel(const AllRows a) {
  all_rows_block<T>(a, blockIdx.x);
}

// A distillation's entry j of a row, the first of its class, where that is one of the columns [col0, col1): what all entries of that class leave of the probability goes to P, and
// what they take from it, negative, to put(col, .).
template <typename Put>
__device__ __forceinline__ void fix_target(const TargetFix& a, int64_t row, int j, int col0, int col1, Put put) {
  const int c = class_of(a.t, row, j, a.classes), col = c - a.first;
  if (c < 0 || col < col0 || col >= col1) return;
  const float2 norm = a.norm[row];
  if (norm.x == INFINITY) return;
  const float given = a.p[row * a.t.k + j];
  if (given < 0.0f) return;
  // the probability less what is given, to a step of the larger one; of the result where both are near 1
  const float d = a.zt[row * a.t.k + j] - norm.x, v = given > 0.5f ? expm1f(d + logf(norm.y)) + (1.0f - given) : expf(d) * norm.y - given;
  if (a.dtype == 1) ((bf16*)a.P)[row * a.ldp + col] = (bf16)v;
  else ((float*)a.P)[row * a.ldp + col] = v;
  if (a.sums) put(col, -given);
}
// Sums in units of 2^-40: integers, so that the order of the additions does not matter.
__device__ __forceinline__ unsigned long long units(float x) { return (unsigned long long)(long long)rint((double)x * 1099511627776.0); }
__device__ __forceinline__ double of_units(unsigned long long u) { return (double)(long long)u * (1.0 / 1099511627776.0); }

__global__ __launch_bounds__(256) void target_fix_kernel(const TargetFix a) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= (int64_t)a.rows * a.t.k) return;
  fix_target(a, at / a.t.k, (int)(at % a.t.k), 0, a.columns, [&](int col, float x) {
    if (x != x) a.sums[col] = NAN;
    else atomicAdd(a.fixed + col, units(x));
  });
}

// 512 columns by 4 EACH rows a workgroup, a lane 8 columns of EACH rows; then, where fix is set, the targets among them.  Workgroups behind those: all_rows_block.  Bound by memory, 4 bytes in, 2 or 4 out:
// 2048 x 32000 bf16 78 us (5.0 TB/s), 1000 x 50001 58 (5.2).
template <typename T, int EACH>
__global__ __launch_bounds__(256) void kept_prob_kernel(const TargetFix a, const float* z, int64_t ldz, const int32_t* labels, bool fix, const AllRows all) {
  constexpr float kLog2e = 1.44269504088896340736f;
  __shared__ float sums[4][512];
  __shared__ unsigned long long fixed[512];
  const int wide = (a.columns + 511) / 512, high = (a.rows + 4 * EACH - 1) / (4 * EACH);
  if ((int)blockIdx.x >= wide * high) {
    all_rows_block<T>(all, blockIdx.x - wide * high);
    return;
  }
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, bx = blockIdx.x % wide, by = blockIdx.x / wide, col0 = bx * 512, c = col0 + lane * 8, row0 = by * 4 * EACH;
  float sum[8] = {};
  if (c < a.columns) {
#pragma unroll 4
    for (int i = 0; i < EACH; ++i) {
      const int row = row0 + w * EACH + i;
      if (row >= a.rows) break;
      const f32x4 u[2] = {*(const f32x4*)(z + row * ldz + c), *(const f32x4*)(z + row * ldz + c + 4)};
      const float2 norm = a.norm[row];
      const int label = labels ? labels[row] - a.first : -1;
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = __builtin_amdgcn_exp2f((u[e / 4][e % 4] - norm.x) * kLog2e) * norm.y;
        if (c + e == label) p[e] = expm1f(u[e / 4][e % 4] - norm.x + logf(norm.y));              // (1 less, and exact where that is near 0)
        if (norm.x == INFINITY || c + e >= a.columns) p[e] = 0.0f;                                // (also where the row holds NaN)
        sum[e] += p[e];
      }
      store8((T*)a.P + (int64_t)row * a.ldp + c, 8, p);
    }
  }
  if (!a.sums && !fix) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[w][lane * 8 + e] = sum[e];
  for (int i = t; i < 512; i += 256) fixed[i] = 0;
  __syncthreads();                       // (what this workgroup has written is in order from here on)
  if (fix) {
    const int rows = a.rows - row0 < 4 * EACH ? a.rows - row0 : 4 * EACH, col1 = col0 + 512 < a.columns ? col0 + 512 : a.columns;
    for (int i = t; i < rows * a.t.k; i += 256)
      fix_target(a, row0 + i / a.t.k, i % a.t.k, col0, col1, [&](int col, float x) {
        if (x != x) sums[0][col - col0] = NAN;
        else atomicAdd(&fixed[col - col0], units(x));
      });
    __syncthreads();
  }
  if (a.sums)
    for (int i = t; i < 512; i += 256)
      if (col0 + i < a.columns)
        a.sums[(int64_t)by * a.columns + col0 + i] = (float)(((double)sums[0][i] + (double)sums[1][i]) + ((double)sums[2][i] + (double)sums[3][i]) + of_units(fixed[i]));
}

template <typename T>
__global__ __launch_bounds__(256) void pad_rows_kernel(const T* in, int64_t ldin, int rows, int cols, T* out, int64_t ldo) {
  const int eights = (cols + 7) / 8;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, row = at / eights;
  const int c = (int)(at % eights) * 8;
  if (row >= rows) return;
  float v[8];
  load8(in + row * ldin + c, cols - c, v);
  store8(out + row * ldo + c, 8, v);
}

// 32 columns a workgroup, 8 strands of parts each, or, of many parts, 8 columns and 32 strands; four loads under way.
template <int COLS>
__device__ __forceinline__ void bias_block(const BiasGradient& a, int block, double (&strand)[256]) {
  constexpr int STRANDS = 256 / COLS;
  const int t = threadIdx.x, l = t % COLS, s = t / COLS, c = block * COLS + l;
  double sum = 0.0;
  if (c < a.columns) {
    int i = s;
    for (; i + 3 * STRANDS < a.parts; i += 4 * STRANDS) {
      float v[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = a.sums[(int64_t)(i + STRANDS * q) * a.columns + c];
      sum += ((double)v[0] + (double)v[1]) + ((double)v[2] + (double)v[3]);
    }
    for (; i < a.parts; i += STRANDS) sum += (double)a.sums[(int64_t)i * a.columns + c];
  }
  strand[t] = sum;
  __syncthreads();
  if (s > 0 || c >= a.columns) return;
  sum = a.fixed ? of_units(a.fixed[c]) : 0.0;
#pragma unroll
  for (int i = 0; i < STRANDS; ++i) sum += strand[i * COLS + l];
  a.dbias[c] = (float)(sum * (double)*a.alpha);
}
__device__ __host__ __forceinline__ bool many_parts(const BiasGradient& a) { return a.parts >= 128; }

// Workgroups behind the joining ones: bias_block.
template <typename T>
__global__ __launch_bounds__(256) void join_parts_kernel(const float* work, int parts, int rows, int cols, const float* alpha, T* out, int64_t ldo, unsigned joins, const BiasGradient bias) {
  if (blockIdx.x >= joins) {
    __shared__ double strand[256];
    if (many_parts(bias)) bias_block<8>(bias, blockIdx.x - joins, strand);
    else bias_block<32>(bias, blockIdx.x - joins, strand);
    return;
  }
  const int quads = (cols + 3) / 4;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, row = at / quads, ldw = (int64_t)quads * 4;
  const int c = (int)(at % quads) * 4;
  if (row >= rows) return;
  f32x4 sum = *(const f32x4*)(work + row * ldw + c);
#pragma unroll 4
  for (int p = 1; p < parts; ++p) sum += *(const f32x4*)(work + ((int64_t)p * rows + row) * ldw + c);
  sum *= *alpha;
  T* const to = out + row * ldo + c;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (c + e < cols) to[e] = (T)sum[e];
}

template <typename T>
__global__ __launch_bounds__(256) void zero_kernel(T* out, int64_t ldo, int rows, int cols) {
  const int eights = (cols + 7) / 8;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, row = at / eights;
  const int c = (int)(at % eights) * 8;
  const float v[8] = {};
  if (row < rows) store8(out + row * ldo + c, cols - c, v);
}

unsigned blocks(int64_t n, int each) { return (unsigned)((n + each - 1) / each); }

}  // namespace

hipError_t launch_target_logits(int dtype, const TargetLogits& a, hipStream_t s) {
  const int64_t targets = (int64_t)a.rows * a.t.k;
  const unsigned n = blocks(targets, 4);
  if (targets <= 1024) {
    if (dtype == 1) target_logits_kernel<bf16, 256><<<(unsigned)targets, 256, 0, s>>>(a);
    else target_logits_kernel<float, 256><<<(unsigned)targets, 256, 0, s>>>(a);
  } else if (a.dim <= 512) {
    const unsigned few = blocks(targets, 16);
    if (dtype == 1) target_logits_kernel<bf16, 16><<<few, 256, 0, s>>>(a);
    else target_logits_kernel<float, 16><<<few, 256, 0, s>>>(a);
  } else if (dtype == 1) target_logits_kernel<bf16, 64><<<n, 256, 0, s>>>(a);
  else target_logits_kernel<float, 64><<<n, 256, 0, s>>>(a);
  return hipGetLastError();
}

// Threads for each row of row_loss_kernel.
static int team_of(const RowLoss& a) {
  if (a.work) return a.classes > 512 ? 256 : 64;
  if (a.rows <= 256) return a.spans > 512 ? 256 : 64;
  return a.t.k > 256 ? 256 : 16;
}
int row_groups(const RowLoss& a) { return (int)blocks(a.rows, 256 / team_of(a)); }
hipError_t launch_row_loss(const RowLoss& a, hipStream_t s) {
  const int team = team_of(a), entries = a.t.top ? 256 / team * (a.t.k | 1) * (int)sizeof(float2) : 0;
  const unsigned grid = (unsigned)row_groups(a) + (a.fixed ? blocks(a.classes, 2048) : 0);
  if (team == 256) row_loss_kernel<256><<<grid, 256, entries, s>>>(a);
  else if (team == 64) row_loss_kernel<64><<<grid, 256, entries, s>>>(a);
  else row_loss_kernel<16><<<grid, 256, entries, s>>>(a);
  return hipGetLastError();
}

// Whether kept_prob_kernel sees to a distillation's targets itself, without `fixed`: as long as its workgroups do not look through too many of them too often.  5184 x 512 with 9:
// additions to `fixed` from all over the chip, 90 to a class, took 9 us more.
bool fixes_targets(int k, int columns) { return k <= 16 || columns <= 2048; }

static unsigned all_rows_blocks(const AllRows& a) { return 1 + (a.xz ? blocks((int64_t)a.rows * ((a.dim + 7) / 8), 256) : 0); }
hipError_t launch_all_rows(int dtype, const AllRows& a, hipStream_t s) {
  if (dtype == 1) all_rows_kernel<bf16><<<all_rows_blocks(a), 256, 0, s>>>(a);
  else all_rows_kernel<float><<<all_rows_blocks(a), 256, 0, s>>>(a);
  return hipGetLastError();
}

// Rows that each wavefront of kept_prob_kernel takes: as few as make 512 workgroups (8192 x 47 24 us with 16, 8 with 4).
static int each_of(int rows, int columns) {
  const int64_t groups = (int64_t)blocks(columns, 512) * rows;
  return groups >= 512 * 64 ? 16 : groups >= 512 * 16 || rows > 4096 ? 4 : 1;
}
int kept_sum_parts(int rows, int columns) { return (int)blocks(rows, 4 * each_of(rows, columns)); }

hipError_t launch_kept_prob(const TargetFix& a, const float* z, int64_t ldz, const int32_t* labels, const AllRows* all, hipStream_t s) {
  // (each workgroup looks through all its rows' targets: few of them, or few workgroups beside each other)
  const bool fix = a.t.top && fixes_targets(a.t.k, a.columns);
  const unsigned grid = blocks(a.columns, 512) * (unsigned)kept_sum_parts(a.rows, a.columns) + (all ? all_rows_blocks(*all) : 0);
  const AllRows more = all ? *all : AllRows{};
  auto launch = [&](auto type, auto each) { kept_prob_kernel<decltype(type), decltype(each)::value><<<grid, 256, 0, s>>>(a, z, ldz, labels, fix, more); };
  auto rows_of = [&](auto type) {
    const int each = each_of(a.rows, a.columns);
    if (each == 16) launch(type, std::integral_constant<int, 16>{});
    else if (each == 4) launch(type, std::integral_constant<int, 4>{});
    else launch(type, std::integral_constant<int, 1>{});
  };
  if (a.dtype == 1) rows_of(bf16{});
  else rows_of(0.0f);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || fix || !a.t.top ? e : launch_target_fix(a, s);
}

hipError_t launch_target_fix(const TargetFix& a, hipStream_t s) {
  target_fix_kernel<<<blocks((int64_t)a.rows * a.t.k, 256), 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_zero(int dtype, void* out, int64_t ldo, int rows, int cols, hipStream_t s) {
  const unsigned n = blocks((int64_t)rows * ((cols + 7) / 8), 256);
  if (dtype == 1) zero_kernel<bf16><<<n, 256, 0, s>>>((bf16*)out, ldo, rows, cols);
  else zero_kernel<float><<<n, 256, 0, s>>>((float*)out, ldo, rows, cols);
  return hipGetLastError();
}

hipError_t launch_pad_rows(int dtype, const void* in, int64_t ldin, int rows, int cols, void* out, int64_t ldo, hipStream_t s) {
  const unsigned n = blocks((int64_t)rows * ((cols + 7) / 8), 256);
  if (dtype == 1) pad_rows_kernel<bf16><<<n, 256, 0, s>>>((const bf16*)in, ldin, rows, cols, (bf16*)out, ldo);
  else pad_rows_kernel<float><<<n, 256, 0, s>>>((const float*)in, ldin, rows, cols, (float*)out, ldo);
  return hipGetLastError();
}

hipError_t launch_join_parts(int dtype, const float* work, int parts, int rows, int cols, const float* alpha, void* out, int64_t ldo, const BiasGradient* bias, hipStream_t s) {
  const unsigned n = blocks((int64_t)rows * ((cols + 3) / 4), 256), more = bias ? blocks(bias->columns, many_parts(*bias) ? 8 : 32) : 0;
  const BiasGradient b = bias ? *bias : BiasGradient{};
  if (dtype == 1) join_parts_kernel<bf16><<<n + more, 256, 0, s>>>(work, parts, rows, cols, alpha, (bf16*)out, ldo, n, b);
  else join_parts_kernel<float><<<n + more, 256, 0, s>>>(work, parts, rows, cols, alpha, (float*)out, ldo, n, b);
  return hipGetLastError();
}

}  // namespace slp
