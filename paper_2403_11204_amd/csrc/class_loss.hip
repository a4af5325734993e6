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
  if (c < 0) {
    if (lane == 0) a.zt[at] = 0.0f;
    return;
  }
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

// 16 rows a workgroup, 16 threads each.
__global__ __launch_bounds__(256) void row_loss_kernel(const RowLoss a) {
  __shared__ float2 part[16][16];
  const int r = threadIdx.x & 15, s = threadIdx.x >> 4;
  const int64_t row = (int64_t)blockIdx.x * 16 + r;
  const bool in = row < a.rows;
  auto all = [&](float2 mine) {           // of the row's 16 threads, in their order
    __syncthreads();
    part[s][r] = mine;
    __syncthreads();
    float2 sum = part[0][r];
    for (int i = 1; i < 16; ++i) sum = joined(sum, part[i][r]);
    return sum;
  };
  auto total = [&](float mine) {
    __syncthreads();
    part[s][r].x = mine;
    __syncthreads();
    float sum = part[0][r].x;
    for (int i = 1; i < 16; ++i) sum += part[i][r].x;
    return sum;
  };
  float2 mine = {-INFINITY, 0.0f};
  if (in)
    for (int i = s; i < a.spans; i += 16) mine = joined(mine, a.stats[(int64_t)i * a.rows + row]);
  mine = all(mine);
  const float log_all = logf(mine.y), lse = mine.x + log_all;         // (apart where the logits are so large that their sum is the largest)
  float loss = 0.0f;
  bool counts = false;
  if (!a.t.top) {
    const int c = in ? class_of(a.t, row, 0, a.classes) : -1;
    counts = c >= 0;
    if (counts && s == 0) loss = log_all + (mine.x - a.zt[row]);
    if (in && s == 0 && a.labels) a.labels[row] = c;
  } else {
    const int k = in ? a.t.k : 0;
    float2 top = {-INFINITY, 0.0f};
    for (int j = s; j < k; j += 16) {
      const float t = teacher(a.t, row, j, a.classes);
      if (t != -INFINITY) top = joined(top, float2{t, 1.0f});
    }
    top = all(top);
    counts = top.y != 0.0f;               // (a NaN counts)
    const float log_sum = logf(top.y);
    for (int j = s; j < k; j += 16) {
      const float t = teacher(a.t, row, j, a.classes);
      const float logp = t - top.x - log_sum, p = counts && t != -INFINITY ? expf(t - top.x) / top.y : 0.0f;
      a.p[row * k + j] = p;
      if (p != 0.0f) loss += p * (logp + log_all + (mine.x - a.zt[row * k + j]));
    }
    loss = total(loss) * a.square_t;
  }
  if (in && s == 0) {
    a.lse[row] = lse;
    a.losses[row] = counts ? loss : 0.0f;
    a.norm[row] = float2{!counts ? INFINITY : mine.x == INFINITY ? NAN : mine.x, 1.0f / mine.y};
  }
}

__global__ __launch_bounds__(1024) void mean_kernel(const float* losses, const float2* norm, int rows, float scale, float* loss, float* alpha) {
  __shared__ double sums[1024];
  __shared__ int counts[1024];
  const int t = threadIdx.x;
  double sum = 0.0;
  int n = 0;
  for (int i = t; i < rows; i += 1024)
    if (norm[i].x != INFINITY) {
      sum += (double)losses[i];
      ++n;
    }
  sums[t] = sum;
  counts[t] = n;
  for (int step = 512; step > 0; step >>= 1) {
    __syncthreads();
    if (t < step) {
      sums[t] += sums[t + step];
      counts[t] += counts[t + step];
    }
  }
  if (t == 0) {
    *loss = counts[0] ? (float)(sums[0] / counts[0]) : 0.0f;
    *alpha = counts[0] ? scale / (float)counts[0] : 0.0f;
  }
}

// The first entry of a class in its row writes what all of that class add up to.
__global__ __launch_bounds__(256) void target_fix_kernel(const TargetFix a) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= (int64_t)a.rows * a.t.k) return;
  const int64_t row = at / a.t.k;
  const int j = (int)(at % a.t.k), c = class_of(a.t, row, j, a.classes), col = c - a.first;
  if (c < 0 || col < 0 || col >= a.columns) return;
  const float2 norm = a.norm[row];
  if (norm.x == INFINITY) return;
  float given = 1.0f;
  if (a.t.top) {
    const float* const p = a.p + row * a.t.k;
    given = 0.0f;
    for (int i = 0; i < a.t.k; ++i)
      if (class_of(a.t, row, i, a.classes) == c) {
        if (i < j) return;
        given += p[i];
      }
  }
  // the probability less what is given, to a step of the larger one; of the result where both are near 1
  const float d = a.zt[at] - norm.x, v = given > 0.5f ? expm1f(d + logf(norm.y)) + (1.0f - given) : expf(d) * norm.y - given;
  if (a.dtype == 1) {
    ((bf16*)a.P)[row * a.ldp + col] = (bf16)v;
  } else {
    ((float*)a.P)[row * a.ldp + col] = v;
  }
  // (integers: the order of the additions does not matter.  One class: the column's sum has left the target out, otherwise it holds the probability.)
  if (a.fixed) {
    const float add = a.t.top ? -given : v;
    if (add != add) a.sums[col] = NAN;
    else atomicAdd(a.fixed + col, (unsigned long long)(long long)rint((double)add * 1099511627776.0));
  }
}

__global__ __launch_bounds__(256) void bias_gradient_kernel(const float* sums, int parts, const unsigned long long* fixed, int columns, const float* alpha, float* dbias) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= columns) return;
  double sum = (double)(long long)fixed[c] * (1.0 / 1099511627776.0);
  for (int i = 0; i < parts; ++i) sum += (double)sums[(int64_t)i * columns + c];
  dbias[c] = (float)(sum * (double)*alpha);
}

__global__ __launch_bounds__(256) void clear_kernel(unsigned long long* p, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = 0;
}

template <typename T>
__global__ __launch_bounds__(256) void pad_rows_kernel(const T* in, int64_t ldin, int rows, int cols, const float2* norm, T* out, int64_t ldo) {
  const int eights = (cols + 7) / 8;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, row = at / eights;
  const int c = (int)(at % eights) * 8;
  if (row >= rows) return;
  float v[8];
  load8(in + row * ldin + c, norm && norm[row].x == INFINITY ? 0 : cols - c, v);
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
  row_loss_kernel<<<blocks(a.rows, 16), 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_mean(const float* losses, const float2* norm, int rows, float scale, float* loss, float* alpha, hipStream_t s) {
  mean_kernel<<<1, 1024, 0, s>>>(losses, norm, rows, scale, loss, alpha);
  return hipGetLastError();
}

hipError_t launch_target_fix(const TargetFix& a, hipStream_t s) {
  target_fix_kernel<<<blocks((int64_t)a.rows * a.t.k, 256), 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_bias_gradient(const float* sums, int parts, const unsigned long long* fixed, int columns, const float* alpha, float* dbias, hipStream_t s) {
  bias_gradient_kernel<<<blocks(columns, 256), 256, 0, s>>>(sums, parts, fixed, columns, alpha, dbias);
  return hipGetLastError();
}

hipError_t launch_clear(unsigned long long* p, int n, hipStream_t s) {
  clear_kernel<<<blocks(n, 256), 256, 0, s>>>(p, n);
  return hipGetLastError();
}

hipError_t launch_zero(int dtype, void* out, int64_t ldo, int rows, int cols, hipStream_t s) {
  const unsigned n = blocks((int64_t)rows * ((cols + 7) / 8), 256);
  if (dtype == 1) zero_kernel<bf16><<<n, 256, 0, s>>>((bf16*)out, ldo, rows, cols);
  else zero_kernel<float><<<n, 256, 0, s>>>((float*)out, ldo, rows, cols);
  return hipGetLastError();
}

hipError_t launch_pad_rows(int dtype, const void* in, int64_t ldin, int rows, int cols, const float2* norm, void* out, int64_t ldo, hipStream_t s) {
  const unsigned n = blocks((int64_t)rows * ((cols + 7) / 8), 256);
  if (dtype == 1) pad_rows_kernel<bf16><<<n, 256, 0, s>>>((const bf16*)in, ldin, rows, cols, norm, (bf16*)out, ldo);
  else pad_rows_kernel<float><<<n, 256, 0, s>>>((const float*)in, ldin, rows, cols, norm, (float*)out, ldo);
  return hipGetLastError();
}

hipError_t launch_join_parts(int dtype, const float* work, int parts, int rows, int cols, const float* alpha, void* out, int64_t ldo, hipStream_t s) {
  const unsigned n = blocks((int64_t)rows * ((cols + 3) / 4), 256);
  if (dtype == 1) join_parts_kernel<bf16><<<n, 256, 0, s>>>(work, parts, rows, cols, alpha, (bf16*)out, ldo);
  else join_parts_kernel<float><<<n, 256, 0, s>>>(work, parts, rows, cols, alpha, (float*)out, ldo);
  return hipGetLastError();
}

}  // namespace slp
