// Losses over the classes of a linear layer: what is done for each row and for each of its targets, around the products in class_products.hip.
//
// With z = x W^T + b, temperature T and a row's targets c(j) of probability p_j (one of probability 1, or a teacher's softmax(top / T)):
//   lse = log sum_v exp(z_v / T)        loss = T^2 sum_j p_j (log p_j + lse - z_c(j) / T)        dz_v = T (exp(z_v / T - lse) - sum of p_j with c(j) = v)
// The logits of the targets are computed apart, in float32: P, which leaves the products rounded to the operands' type, gets exp(z_c / T - lse) - p_j written over
// it, so that nothing cancels among rounded values.
#include "class_loss.h"
#include "eightbit_device.h"

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
  if (class_of(t, row, j, classes) < 0) return -INFINITY;
  const int64_t at = row * t.ldtop + j;
  return (t.top_dtype == 1 ? (float)((const bf16*)t.top)[at] : ((const float*)t.top)[at]) * t.per_t;
}

// One wavefront for each target: the dot product of a row of x and the row of W that is its class.  Bound by reading those rows of W: 4096 x 64
// targets of 4096 bf16 are 2.1 GB.
template <typename T>
__global__ __launch_bounds__(256) void target_logits_kernel(const TargetLogits a) {
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (at >= (int64_t)a.rows * a.t.k) return;
  const int64_t row = at / a.t.k;
  const int c = class_of(a.t, row, (int)(at % a.t.k), a.classes);
  if (c < a.kept) return;                // (none, or kept)
  const T* const x = (const T*)a.x + row * a.ldx;
  const T* const w = (const T*)a.w + (int64_t)c * a.ldw;
  float sum = 0.0f;
  for (int d = lane * 8; d < a.dim; d += 512) {
    float u[8], v[8];
    load8(x + d, a.dim - d, u);
    load8(w + d, a.dim - d, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += u[e] * v[e];
  }
  sum = sum_of_64(sum);
  if (lane == 0) a.zt[at] = (sum + (a.bias ? a.bias[c] : 0.0f)) * a.t.per_t;
}

// (largest, sum of exp(z - largest)) of two sets together; the largest of nothing is -infinity
__device__ __forceinline__ float2 joined(float2 a, float2 b) {
  const float most = fmaxf(a.x, b.x);
  return float2{most, (a.x == most ? a.y : a.y * expf(a.x - most)) + (b.x == most ? b.y : b.y * expf(b.x - most))};
}

// TEAM threads a row: 16, or all 256 of a workgroup where there are few rows (1 x 131072 classes, 1024 spans: 35 us on 16 threads).
template <int TEAM>
__global__ __launch_bounds__(256) void row_loss_kernel(const RowLoss a) {
  constexpr int ROWS = 256 / TEAM;
  __shared__ float2 part[TEAM][ROWS];
  extern __shared__ float2 entries[];          // of a distillation: class and probability of each row's entries
  const int r = threadIdx.x % ROWS, s = threadIdx.x / ROWS;
  const int64_t row = (int64_t)blockIdx.x * ROWS + r;
  const bool in = row < a.rows;
  // of the row's threads, halves of them at a time: the same order every time
  auto all = [&](float2 mine) {
    __syncthreads();
    part[s][r] = mine;
    for (int step = TEAM / 2; step > 0; step >>= 1) {
      __syncthreads();
      if (s < step) part[s][r] = joined(part[s][r], part[s + step][r]);
    }
    __syncthreads();
    return part[0][r];
  };
  auto total = [&](float mine) {
    __syncthreads();
    part[s][r].x = mine;
    for (int step = TEAM / 2; step > 0; step >>= 1) {
      __syncthreads();
      if (s < step) part[s][r].x += part[s + step][r].x;
    }
    __syncthreads();
    return part[0][r].x;
  };
  float2 mine = {-INFINITY, 0.0f};
  if (in) {
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
    for (int j = s; j < k; j += TEAM) {
      const float t = teacher(a.t, row, j, a.classes);
      if (t != -INFINITY) top = joined(top, float2{t, 1.0f});
    }
    top = all(top);
    counts = top.y != 0.0f;               // (a NaN counts)
    const float log_sum = logf(top.y);
    for (int j = s; j < k; j += TEAM) {
      const int c = class_of(a.t, row, j, a.classes);
      const float t = teacher(a.t, row, j, a.classes), z = c >= 0 ? logit(j, c) : 0.0f;
      const float logp = t - top.x - log_sum, p = counts && t != -INFINITY ? expf(t - top.x) / top.y : 0.0f;
      entries[r * (k | 1) + j] = float2{__builtin_bit_cast(float, c), p};
      if (p != 0.0f) loss += p * (logp + log_all + (mine.x - z));
    }
    loss = total(loss) * a.square_t;
    // what the entries of one class add up to, at the first of them
    for (int j = s; j < k; j += TEAM) {
      const int c = __builtin_bit_cast(int, entries[r * (k | 1) + j].x);
      float sum = 0.0f;
      bool first = true;
      for (int i = 0; i < k; ++i) {
        const float2 e = entries[r * (k | 1) + i];
        if (__builtin_bit_cast(int, e.x) == c) {
          sum += e.y;
          first &= i >= j;
        }
      }
      a.p[row * k + j] = first ? sum : -1.0f;
    }
  }
  if (in && s == 0) {
    a.lse[row] = lse;
    a.losses[row] = counts ? loss : 0.0f;
    a.norm[row] = float2{!counts ? INFINITY : mine.x == INFINITY ? NAN : mine.x, 1.0f / mine.y};
  }
}

// Workgroup 0: the mean.  The others: 2048 elements each of xz's rows, then of `fixed`.
template <typename T>
__global__ __launch_bounds__(256) void all_rows_kernel(const AllRows a, int pads) {
  const int t = threadIdx.x;
  if (blockIdx.x == 0) {
    __shared__ double sums[256];
    __shared__ int counts[256];
    double sum = 0.0;
    int n = 0;
    for (int i0 = t; i0 < a.rows; i0 += 2048) {         // eight loads under way
      float loss[8], peak[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int i = i0 + 256 * q;
        loss[q] = i < a.rows ? a.losses[i] : 0.0f;
        peak[q] = i < a.rows ? a.norm[i].x : INFINITY;
      }
#pragma unroll
      for (int q = 0; q < 8; ++q)
        if (peak[q] != INFINITY) {
          sum += (double)loss[q];
          ++n;
        }
    }
    sums[t] = sum;
    counts[t] = n;
    for (int step = 128; step > 0; step >>= 1) {
      __syncthreads();
      if (t < step) {
        sums[t] += sums[t + step];
        counts[t] += counts[t + step];
      }
    }
    if (t == 0) {
      *a.loss = counts[0] ? (float)(sums[0] / counts[0]) : 0.0f;
      *a.alpha = counts[0] ? a.scale / (float)counts[0] : 0.0f;
    }
    return;
  }
  const int64_t at = (int64_t)(blockIdx.x - 1) * 256 + t;
  if ((int)blockIdx.x <= pads) {
    const int eights = (a.dim + 7) / 8;
    const int64_t row = at / eights;
    const int c = (int)(at % eights) * 8;
    if (row >= a.rows) return;
    float v[8];
    load8((const T*)a.x + row * a.ldx + c, a.norm[row].x == INFINITY ? 0 : a.dim - c, v);
    store8((T*)a.xz + row * a.ldxz + c, 8, v);
    return;
  }
  const int64_t i = (at - (int64_t)pads * 256) * 8;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (i + e < a.classes) a.fixed[i + e] = 0;
}

// Entry j of a row, the first of its class, where that is one of the columns [col0, col1).
// sums: a part of the columns' sums that is there already.
__device__ __forceinline__ void fix_target(const TargetFix& a, int64_t row, int j, int col0, int col1, float* sums) {
  const int c = class_of(a.t, row, j, a.classes), col = c - a.first;
  if (c < 0 || col < col0 || col >= col1) return;
  const float2 norm = a.norm[row];
  if (norm.x == INFINITY) return;
  const float given = a.t.top ? a.p[row * a.t.k + j] : 1.0f;
  if (given < 0.0f) return;
  // the probability less what is given, to a step of the larger one; of the result where both are near 1
  const float d = a.zt[row * a.t.k + j] - norm.x, v = given > 0.5f ? expm1f(d + logf(norm.y)) + (1.0f - given) : expf(d) * norm.y - given;
  if (a.dtype == 1) ((bf16*)a.P)[row * a.ldp + col] = (bf16)v;
  else ((float*)a.P)[row * a.ldp + col] = v;
  // (integers: the order of the additions does not matter.  One class: the column's sum has left the target out, otherwise it holds the probability.)
  if (a.fixed) {
    const float add = a.t.top ? -given : v;
    if (add != add) sums[col] = NAN;
    else atomicAdd(a.fixed + col, (unsigned long long)(long long)rint((double)add * 1099511627776.0));
  }
}

__global__ __launch_bounds__(256) void target_fix_kernel(const TargetFix a) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at < (int64_t)a.rows * a.t.k) fix_target(a, at / a.t.k, (int)(at % a.t.k), 0, a.columns, a.sums);
}

// 512 columns by 4 EACH rows a workgroup, a lane 8 columns of EACH rows; then, where fix is set, the targets among them.  Bound by memory: 4 bytes in, 2 or 4 out.
template <typename T, int EACH>
__global__ __launch_bounds__(256) void kept_prob_kernel(const TargetFix a, const float* z, int64_t ldz, const int32_t* labels, bool fix) {
  constexpr float kLog2e = 1.44269504088896340736f;
  __shared__ float sums[4][512];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, col0 = blockIdx.x * 512, c = col0 + lane * 8, row0 = blockIdx.y * 4 * EACH;
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
        if (norm.x == INFINITY || c + e == label || c + e >= a.columns) p[e] = 0.0f;       // (also where the row holds NaN)
        sum[e] += p[e];
      }
      store8((T*)a.P + (int64_t)row * a.ldp + c, 8, p);
    }
  }
  if (a.sums) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[w][lane * 8 + e] = sum[e];
  }
  __syncthreads();                       // (what this workgroup has written is in order from here on)
  if (a.sums) {
    for (int i = t; i < 512; i += 256)
      if (col0 + i < a.columns) a.sums[(int64_t)blockIdx.y * a.columns + col0 + i] = (sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]);
    __syncthreads();
  }
  if (!fix) return;
  const int rows = a.rows - row0 < 4 * EACH ? a.rows - row0 : 4 * EACH, col1 = col0 + 512 < a.columns ? col0 + 512 : a.columns;
  for (int i = t; i < rows * a.t.k; i += 256) fix_target(a, row0 + i / a.t.k, i % a.t.k, col0, col1, a.sums + (int64_t)blockIdx.y * a.columns);
}

// 32 columns a workgroup, 8 strands of parts each, four loads under way.
__global__ __launch_bounds__(256) void bias_gradient_kernel(const float* sums, int parts, const unsigned long long* fixed, int columns, const float* alpha, float* dbias) {
  __shared__ double strand[8][32];
  const int t = threadIdx.x, l = t & 31, s = t >> 5, c = blockIdx.x * 32 + l;
  double sum = 0.0;
  if (c < columns) {
    int i = s;
    for (; i + 24 < parts; i += 32) {
      float v[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = sums[(int64_t)(i + 8 * q) * columns + c];
      sum += ((double)v[0] + (double)v[1]) + ((double)v[2] + (double)v[3]);
    }
    for (; i < parts; i += 8) sum += (double)sums[(int64_t)i * columns + c];
  }
  strand[s][l] = sum;
  __syncthreads();
  if (s > 0 || c >= columns) return;
  sum = (double)(long long)fixed[c] * (1.0 / 1099511627776.0);
  for (int i = 0; i < 8; ++i) sum += strand[i][l];
  dbias[c] = (float)(sum * (double)*alpha);
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

template <typename T>
__global__ __launch_bounds__(256) void join_parts_kernel(const float* work, int parts, int rows, int cols, const float* alpha, T* out, int64_t ldo) {
  const int quads = (cols + 3) / 4;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, row = at / quads, ldw = (int64_t)quads * 4;
  const int c = (int)(at % quads) * 4;
  if (row >= rows) return;
  f32x4 sum = *(const f32x4*)(work + row * ldw + c);
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
  const unsigned n = blocks((int64_t)a.rows * a.t.k, 4);
  if (dtype == 1) target_logits_kernel<bf16><<<n, 256, 0, s>>>(a);
  else target_logits_kernel<float><<<n, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_row_loss(const RowLoss& a, hipStream_t s) {
  const int entries = a.t.top ? (a.t.k | 1) * (int)sizeof(float2) : 0;
  if (a.rows <= 256 || a.t.k > 256) row_loss_kernel<256><<<a.rows, 256, entries, s>>>(a);
  else row_loss_kernel<16><<<blocks(a.rows, 16), 256, 16 * entries, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_all_rows(int dtype, const AllRows& a, hipStream_t s) {
  const unsigned pads = a.xz ? blocks((int64_t)a.rows * ((a.dim + 7) / 8), 256) : 0, clears = a.fixed ? blocks(a.classes, 2048) : 0;
  if (dtype == 1) all_rows_kernel<bf16><<<1 + pads + clears, 256, 0, s>>>(a, (int)pads);
  else all_rows_kernel<float><<<1 + pads + clears, 256, 0, s>>>(a, (int)pads);
  return hipGetLastError();
}

// Rows of a workgroup of kept_prob_kernel: few where there are few, so that there are workgroups.
int kept_sum_parts(int rows) { return (int)blocks(rows, rows >= 1024 ? 64 : 16); }

hipError_t launch_kept_prob(const TargetFix& a, const float* z, int64_t ldz, const int32_t* labels, hipStream_t s) {
  // each workgroup looks through its rows' targets: a few of them
  const bool fix = a.t.k <= 16;
  const dim3 grid(blocks(a.columns, 512), kept_sum_parts(a.rows));
  if (a.rows >= 1024) {
    if (a.dtype == 1) kept_prob_kernel<bf16, 16><<<grid, 256, 0, s>>>(a, z, ldz, labels, fix);
    else kept_prob_kernel<float, 16><<<grid, 256, 0, s>>>(a, z, ldz, labels, fix);
  } else {
    if (a.dtype == 1) kept_prob_kernel<bf16, 4><<<grid, 256, 0, s>>>(a, z, ldz, labels, fix);
    else kept_prob_kernel<float, 4><<<grid, 256, 0, s>>>(a, z, ldz, labels, fix);
  }
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || fix ? e : launch_target_fix(a, s);
}

hipError_t launch_target_fix(const TargetFix& a, hipStream_t s) {
  target_fix_kernel<<<blocks((int64_t)a.rows * a.t.k, 256), 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_bias_gradient(const float* sums, int parts, const unsigned long long* fixed, int columns, const float* alpha, float* dbias, hipStream_t s) {
  bias_gradient_kernel<<<blocks(columns, 32), 256, 0, s>>>(sums, parts, fixed, columns, alpha, dbias);
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

hipError_t launch_join_parts(int dtype, const float* work, int parts, int rows, int cols, const float* alpha, void* out, int64_t ldo, hipStream_t s) {
  const unsigned n = blocks((int64_t)rows * ((cols + 3) / 4), 256);
  if (dtype == 1) join_parts_kernel<bf16><<<n, 256, 0, s>>>(work, parts, rows, cols, alpha, (bf16*)out, ldo);
  else join_parts_kernel<float><<<n, 256, 0, s>>>(work, parts, rows, cols, alpha, (float*)out, ldo);
  return hipGetLastError();
}

}  // namespace slp
