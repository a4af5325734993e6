// Root-mean-square norm with the residual's addition, its output also in 8 bits with a scale for each 128 elements, and its backward
// pass.
//
//   h = x + r (rounded to the type: the norm is of what is stored);  n = 1 / sqrt(mean(h^2) + eps);  y = h n gamma
//   dx_j = dh_j + n (gamma_j dy_j - h_j n^2 mean(gamma dy h));  dgamma_j = sum over the rows of dy_j h_j n
//
// Sums and everything between the loads and the stores are float32.
#include "eightbit_device.h"

namespace slp {
namespace {

// A chunk is 8 consecutive columns, the columns of a scale are 16 lanes'.  WAVES wavefronts share a row, each lane CH chunks of it in
// registers; MANY: rows longer than that, read twice.
template <typename T, int WAVES, int CH, bool MANY>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void rmsnorm_kernel(const NormArgs a) {
  constexpr int TEAM = WAVES * 64, ROWS = WAVES == 1 ? 4 : 1;
  __shared__ float part[WAVES];
  const int t = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t row = (int64_t)blockIdx.x * ROWS + (WAVES == 1 ? threadIdx.x >> 6 : 0);
  if (row >= a.rows) return;           // (a whole wavefront, and no barrier where a workgroup holds several rows)
  const T* x = (const T*)a.x + row * a.ldx;
  const T* r = a.r ? (const T*)a.r + row * a.ldr : nullptr;
  T* h = a.h ? (T*)a.h + row * a.ldh : nullptr;
  const int D = a.dim;
  const int padded = (D + 127) / 128 * 16;        // chunks, the last scale's whole

  float v[CH][8];
  float ss = 0.0f;
  auto load = [&](int c, float (&o)[8]) {
    load8(x + 8 * c, D - 8 * c, o);
    if (r) {
      float u[8];
      load8(r + 8 * c, D - 8 * c, u);
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = (float)(T)(o[j] + u[j]);
    }
  };
  for (int c0 = 0; c0 < padded; c0 += CH * TEAM) {
#pragma unroll
    for (int i = 0; i < CH; ++i) load(c0 + i * TEAM + t, v[i]);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = c0 + i * TEAM + t;
      if (h) store8(h + 8 * c, D - 8 * c, v[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) ss += v[i][j] * v[i][j];
    }
    if (!MANY) break;
  }
  ss = sum_of_64(ss);
  if (WAVES > 1) {
    if ((t & 63) == 0) part[t >> 6] = ss;
    __syncthreads();
    ss = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) ss += part[w];
  }
  const float n = 1.0f / sqrtf(ss / (float)D + a.eps);
  if (a.rstd && t == 0) a.rstd[row] = n;
  if (!a.y && !a.q) return;
  for (int c0 = 0; c0 < padded; c0 += CH * TEAM) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = c0 + i * TEAM + t;
      if (MANY) {
        if (h) load8(h + 8 * c, D - 8 * c, v[i]);
        else load(c, v[i]);
      }
      float g[8];
      uint32_t amax = 0;
      if (a.gamma) load8(a.gamma + 8 * c, D - 8 * c, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[i][j] *= n;
        if (a.gamma) v[i][j] *= g[j];
        if (8 * c + j >= D) v[i][j] = 0.0f;           // (0 times an infinite n)
        amax = umax(amax, magnitude(v[i][j]));
      }
      if (a.y) store8((T*)a.y + row * a.ldy + 8 * c, D - 8 * c, v[i]);
      if (a.q) {
        const uint32_t scale = scale_of(max_of_16(amax));
        const float up = inverse_scale(scale);
        if (8 * c < ((D + 15) & ~15))                 // zeros up to the next 16 bytes
          *(u32x2*)(a.q + row * a.ldq + 8 * c) = u32x2{to_e4m3(v[i][0] * up, v[i][1] * up, v[i][2] * up, v[i][3] * up),
                                                      to_e4m3(v[i][4] * up, v[i][5] * up, v[i][6] * up, v[i][7] * up)};
        if ((t & 15) == 0 && 8 * c < D) a.scales[row * a.lds + c / 16] = (uint8_t)scale;
      }
    }
    if (!MANY) break;
  }
}

template <typename T>
hipError_t rmsnorm_of(const NormArgs& a, hipStream_t s) {
  const dim3 quads((a.rows + 3) / 4), rows(a.rows);
  if (a.dim <= 512) rmsnorm_kernel<T, 1, 1, false><<<quads, 256, 0, s>>>(a);
  else if (a.dim <= 1024) rmsnorm_kernel<T, 1, 2, false><<<quads, 256, 0, s>>>(a);
  else if (a.dim <= 2048) rmsnorm_kernel<T, 4, 1, false><<<rows, 256, 0, s>>>(a);
  else if (a.dim <= 4096) rmsnorm_kernel<T, 4, 2, false><<<rows, 256, 0, s>>>(a);
  else if (a.dim <= 8192) rmsnorm_kernel<T, 8, 2, false><<<rows, 512, 0, s>>>(a);
  else if (a.dim <= 16384) rmsnorm_kernel<T, 8, 4, false><<<rows, 512, 0, s>>>(a);
  else rmsnorm_kernel<T, 16, 2, true><<<rows, 1024, 0, s>>>(a);
  return hipGetLastError();
}

// ---- backward, any width: the rows' products first, then the columns --------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void rmsnorm_dots_kernel(const NormBackArgs a, float* dots) {
  __shared__ float part[4];
  const int64_t row = blockIdx.x;
  const T *dy = (const T*)a.dy + row * a.lddy, *h = (const T*)a.h + row * a.ldh;
  float dot = 0.0f;
  for (int c = threadIdx.x; 8 * c < a.dim; c += 256) {
    float y[8], x[8], g[8];
    load8(dy + 8 * c, a.dim - 8 * c, y);
    load8(h + 8 * c, a.dim - 8 * c, x);
    if (a.gamma) load8(a.gamma + 8 * c, a.dim - 8 * c, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) dot += (a.gamma ? g[j] : 1.0f) * y[j] * x[j];
  }
  dot = sum_of_64(dot);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = dot;
  __syncthreads();
  if (threadIdx.x == 0) {
    const float n = a.rstd[row];
    dots[row] = n * n * ((part[0] + part[1]) + (part[2] + part[3])) / (float)a.dim;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void rmsnorm_columns_kernel(const NormBackArgs a, const float* dots, float* partials) {
  const int c = 8 * (blockIdx.x * 256 + threadIdx.x), left = a.dim - c;
  if (left <= 0) return;
  float g[8], acc[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    g[j] = 1.0f;
    acc[j] = 0.0f;
  }
  if (a.gamma) load8(a.gamma + c, left, g);
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    float y[8], x[8], d[8];
    const float n = a.rstd[row], k = dots[row];
    load8((const T*)a.dy + row * a.lddy + c, left, y);
    load8((const T*)a.h + row * a.ldh + c, left, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) d[j] = 0.0f;
    if (a.dh) load8((const T*)a.dh + row * a.lddh + c, left, d);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      acc[j] += y[j] * x[j] * n;
      d[j] += n * (g[j] * y[j] - x[j] * k);
    }
    store8((T*)a.dx + row * a.lddx + c, left, d);
  }
  if (a.dgamma) store8(partials + (int64_t)blockIdx.y * a.dim + c, left, acc);
}

int column_groups(int rows) { return rows < 256 ? rows : 256; }

template <typename T>
hipError_t rmsnorm_backward_of(const NormBackArgs& a, hipStream_t s) {
  float *dots = a.work, *partials = a.work + (a.rows + 3) / 4 * 4;
  rmsnorm_dots_kernel<T><<<a.rows, 256, 0, s>>>(a, dots);
  const int groups = column_groups(a.rows);
  rmsnorm_columns_kernel<T><<<dim3((a.dim + 2047) / 2048, groups), 256, 0, s>>>(a, dots, partials);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.dgamma) return e;
  return launch_sum_rows(partials, groups, a.dim, a.dgamma, s);
}

// One column a thread of 64, 4 strands of rows.
__global__ __launch_bounds__(256) void sum_rows_kernel(const float* __restrict__ in, int n, int cols, float* __restrict__ out) {
  __shared__ float part[4][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), strand = threadIdx.x >> 6;
  float sum = 0.0f;
  if (c < cols)
    for (int i = strand; i < n; i += 4) sum += in[(int64_t)i * cols + c];
  part[strand][threadIdx.x & 63] = sum;
  __syncthreads();
  if (strand == 0 && c < cols) out[c] = (part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]);
}

}  // namespace

hipError_t launch_sum_rows(const float* in, int n, int cols, float* out, hipStream_t s) {
  sum_rows_kernel<<<(cols + 63) / 64, 256, 0, s>>>(in, n, cols, out);
  return hipGetLastError();
}

hipError_t launch_rmsnorm(int dtype, const NormArgs& a, hipStream_t s) { return dtype == 1 ? rmsnorm_of<bf16>(a, s) : rmsnorm_of<float>(a, s); }

size_t rmsnorm_backward_floats(int rows, int dim) { return (size_t)((rows + 3) / 4 * 4) + (size_t)column_groups(rows) * dim; }

hipError_t launch_rmsnorm_backward(int dtype, const NormBackArgs& a, hipStream_t s) {
  return dtype == 1 ? rmsnorm_backward_of<bf16>(a, s) : rmsnorm_backward_of<float>(a, s);
}

}  // namespace slp
