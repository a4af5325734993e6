// Root-mean-square norm with the residual's addition, its output also in 8 bits with a scale for each 128 elements, and its backward
// pass.
//
//   h = x + r (rounded to the type: the norm is of what is stored);  n = 1 / sqrt(mean(h^2) + eps);  y = h n gamma
//   dx_j = dh_j + n (gamma_j dy_j - h_j n^2 mean(gamma dy h));  dgamma_j = sum over the rows of dy_j h_j n
//
// Sums and everything between the loads and the stores are float32.  The backward pass takes h as h n, which is of the size of one, in every product: dy h, n^2 and n^3 may
// leave float32's range where dx and dgamma do not.
#include "eightbit_device.h"

namespace slp {
namespace {

// A chunk is 8 consecutive columns, the columns of a scale are 16 lanes'.  What follows the row's rstd n, for one chunk (v: h, g: gamma).
template <typename T>
__device__ __forceinline__ void finish_chunk(const NormArgs& a, int64_t row, int c, float n, const float (&g)[8], float (&v)[8]) {
  const int D = a.dim;
  uint32_t amax = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    v[j] = 8 * c + j < D ? v[j] * n * g[j] : 0.0f;        // (0 times an infinite n)
    amax = umax(amax, magnitude(v[j]));
  }
  if (a.y) store8((T*)a.y + row * a.ldy + 8 * c, D - 8 * c, v);
  if (a.q) {
    const uint32_t scale = scale_of(max_of_16(amax));
    if (8 * c < ((D + 15) & ~15)) *(u32x2*)(a.q + row * a.ldq + 8 * c) = to_e4m3(v, scale_value(scale));      // zeros up to the next 16 bytes
    if ((threadIdx.x & 15) == 0 && 8 * c < D) a.scales[row * a.lds + c / 16] = (uint8_t)scale;
  }
}

// Rows dealt out to teams of WAVES wavefronts, each lane CH chunks of a row in registers; the next row's loads are under way while this one is
// added up and stored.  Bound by memory: 8192 x 16384 bf16 with the residual 173 us (939 MB, 5.4 TB/s), 4096 x 8192 39 us (235 MB), on 512
// workgroups of 8 or 16 wavefronts; a workgroup for each row 181 and 49 us, 256 workgroups 171 and 45 (8192 x 4096 45 -> 59), 1024 177 and 45.  Teams of 4 wavefronts
// on 1024 workgroups: 5000 x 1500 14.2 us, 19.7 on 512; 8192 x 2048 21.5, 23.8.  A team holds little more than its rows: 2000 x 9000 in 3 chunks of 8
// wavefronts 27.3, in 4 45.6, in 2 of 16 36.6; 4096 x 16384 float32 in 2 chunks of 16 wavefronts 165, in 4 of 8 172, one row 5.4 and 6.3.
// Rows of up to 128 (256, where there are many) on LANES = 16: 8192 x 64 3.8 us, on whole wavefronts 6.2; 100000 x 128 16.2, 43.1; 16384 x 80 float32 5.4, 9.3; 8192 x 200 5.5,
// 6.8, but 1000 x 129 4.1, 3.3.
template <typename T, int WAVES, int CH, int LANES = 64>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void rmsnorm_kernel(const NormArgs a) {
  constexpr int TEAM = WAVES * LANES, TEAMS = WAVES == 1 ? 256 / LANES : 1;
  __shared__ float part[2][WAVES];
  const int t = WAVES == 1 ? threadIdx.x % LANES : threadIdx.x, D = a.dim, step = gridDim.x * TEAMS;
  float g[CH][8];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j) g[i][j] = 1.0f;
    if (a.gamma) load8(a.gamma + 8 * (i * TEAM + t), D - 8 * (i * TEAM + t), g[i]);
  }
  Raw<T> x[CH], r[CH];
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = 8 * (i * TEAM + t);
      fetch8((const T*)a.x + row * a.ldx + c, D - c, x[i]);
      if (a.r) fetch8((const T*)a.r + row * a.ldr + c, D - c, r[i]);
    }
  };
  int64_t row = (int64_t)blockIdx.x * TEAMS + (WAVES == 1 ? threadIdx.x / LANES : 0);
  if (row < a.rows) fetch(row);
  for (int turn = 0; row < a.rows; row += step, turn ^= 1) {
    float v[CH][8], ss = 0.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = 8 * (i * TEAM + t);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[i][j] = item(x[i], j);
        if (a.r) v[i][j] = (float)(T)(v[i][j] + item(r[i], j));
        ss += v[i][j] * v[i][j];
      }
      if (a.h) store8((T*)a.h + row * a.ldh + c, D - c, v[i]);
    }
    if (row + step < a.rows) fetch(row + step);
    ss = LANES == 16 ? sum_of_16(ss) : sum_of_64(ss);
    if (WAVES > 1) {
      if ((t & 63) == 0) part[turn][t >> 6] = ss;
      __syncthreads();
      ss = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) ss += part[turn][w];
    }
    const float n = 1.0f / sqrtf(ss / (float)D + a.eps);
    if (a.rstd && t == 0) a.rstd[row] = n;
    if (a.y || a.q) {
#pragma unroll
      for (int i = 0; i < CH; ++i) finish_chunk<T>(a, row, i * TEAM + t, n, g[i], v[i]);
    }
  }
}

constexpr int kOnePass = 16384;       // longest row that a workgroup's registers hold

// Longer rows, read twice: a workgroup of 16 wavefronts for each.
template <typename T>
__global__ __launch_bounds__(1024) void rmsnorm_long_kernel(const NormArgs a) {
  __shared__ float part[16];
  const int64_t row = blockIdx.x;
  const int D = a.dim, chunks = (D + 127) / 128 * 16;
  const T* x = (const T*)a.x + row * a.ldx;
  const T* r = a.r ? (const T*)a.r + row * a.ldr : nullptr;
  T* h = a.h ? (T*)a.h + row * a.ldh : nullptr;
  auto load = [&](int c, float (&o)[8]) {
    load8(x + 8 * c, D - 8 * c, o);
    if (r) {
      float u[8];
      load8(r + 8 * c, D - 8 * c, u);
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = (float)(T)(o[j] + u[j]);
    }
  };
  float ss = 0.0f;
  for (int c = threadIdx.x; c < chunks; c += 1024) {
    float v[8];
    load(c, v);
    if (h) store8(h + 8 * c, D - 8 * c, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) ss += v[j] * v[j];
  }
  ss = sum_of_64(ss);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = ss;
  __syncthreads();
  ss = 0.0f;
#pragma unroll
  for (int w = 0; w < 16; ++w) ss += part[w];
  const float n = 1.0f / sqrtf(ss / (float)D + a.eps);
  if (a.rstd && threadIdx.x == 0) a.rstd[row] = n;
  if (!a.y && !a.q) return;
  for (int c = threadIdx.x; c < chunks; c += 1024) {
    float v[8], g[8] = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f};
    if (h) load8(h + 8 * c, D - 8 * c, v);
    else load(c, v);
    if (a.gamma) load8(a.gamma + 8 * c, D - 8 * c, g);
    finish_chunk<T>(a, row, c, n, g, v);
  }
}

template <typename T>
hipError_t rmsnorm_of(const NormArgs& a, hipStream_t s) {
  const int quads = (a.rows + 3) / 4, few = quads < 2048 ? quads : 2048, sixteens = (quads + 3) / 4 < 2048 ? (quads + 3) / 4 : 2048, rows = a.rows < 512 ? a.rows : 512, twice = a.rows < 1024 ? a.rows : 1024;
  if (a.dim <= 128) rmsnorm_kernel<T, 1, 1, 16><<<sixteens, 256, 0, s>>>(a);
  else if (a.dim <= 256 && a.rows >= 4096) rmsnorm_kernel<T, 1, 2, 16><<<sixteens, 256, 0, s>>>(a);
  else if (a.dim <= 512) rmsnorm_kernel<T, 1, 1><<<few, 256, 0, s>>>(a);
  else if (a.dim <= 1024) rmsnorm_kernel<T, 1, 2><<<few, 256, 0, s>>>(a);
  else if (a.dim <= 2048) rmsnorm_kernel<T, 4, 1><<<twice, 256, 0, s>>>(a);
  else if (a.dim <= 4096) rmsnorm_kernel<T, 4, 2><<<twice, 256, 0, s>>>(a);
  else if (a.dim <= 8192) rmsnorm_kernel<T, 8, 2><<<rows, 512, 0, s>>>(a);
  else if (a.dim <= 12288) rmsnorm_kernel<T, 8, 3><<<rows, 512, 0, s>>>(a);
  else if (a.dim <= kOnePass) rmsnorm_kernel<T, 16, 2><<<rows, 1024, 0, s>>>(a);
  else rmsnorm_long_kernel<T><<<a.rows, 1024, 0, s>>>(a);
  return hipGetLastError();
}

// ---- backward: rows dealt out to teams of WAVES wavefronts, gamma and the sums for its gradient in registers, each lane CH chunks ----
// One reading of everything: a row waits in registers for its product, while the next row's loads are under way (AHEAD; 16 wavefronts have no registers
// for it).  Bound by memory: 4096 x 8192 bf16 with the gradient past the norm 49 us (268 MB, 5.5 TB/s), and 5 for the sums over the workgroups; rows of 8193 to
// 16384 in 2 chunks of 16 wavefronts 4096 x 16384 108 us with the sums, 1 x 16384 4.7, in 4 of 8 wavefronts 112 and 6.1.  Up to 256 on LANES = 16: 100000 x 128 19.6 us, on whole wavefronts 44.6; 16384 x 80
// float32 8.6, 12.5; 1410 x 80 5.7, 6.5; 8192 x 200 8.2, 10.4.
template <typename T, int WAVES, int CH, bool AHEAD, int LANES = 64>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void rmsnorm_backward_kernel(const NormBackArgs a, float* __restrict__ partials) {
  constexpr int TEAM = WAVES * LANES, TEAMS = WAVES == 1 ? 256 / LANES : 1;
  __shared__ float part[2][WAVES];
  __shared__ float sums[TEAMS][WAVES == 1 ? CH * TEAM * 8 : 1];
  const int t = WAVES == 1 ? threadIdx.x % LANES : threadIdx.x, team = WAVES == 1 ? threadIdx.x / LANES : 0;
  const int D = a.dim, step = gridDim.x * TEAMS;
  const float over = 1.0f / (float)D;
  float g[CH][8], acc[CH][8];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = 8 * (i * TEAM + t);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      g[i][j] = 1.0f;
      acc[i][j] = 0.0f;
    }
    if (a.gamma) load8(a.gamma + c, D - c, g[i]);
  }
  Raw<T> y[CH], x[CH], d[CH];
  auto fetch = [&](int64_t row, Raw<T>(&y)[CH], Raw<T>(&x)[CH], Raw<T>(&d)[CH]) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = 8 * (i * TEAM + t);
      fetch8((const T*)a.dy + row * a.lddy + c, D - c, y[i]);
      fetch8((const T*)a.h + row * a.ldh + c, D - c, x[i]);
      if (a.dh) fetch8((const T*)a.dh + row * a.lddh + c, D - c, d[i]);
    }
  };
  int64_t row = (int64_t)blockIdx.x * TEAMS + team;
  if (AHEAD && row < a.rows) fetch(row, y, x, d);
  for (int turn = 0; row < a.rows; row += step, turn ^= 1) {
    if (!AHEAD) fetch(row, y, x, d);
    const float n = a.rstd[row];
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float xn = item(x[i], j) * n;
        dot += g[i][j] * item(y[i], j) * xn;
        acc[i][j] += item(y[i], j) * xn;
      }
    Raw<T> y2[CH], x2[CH], d2[CH];
    if (AHEAD && row + step < a.rows) fetch(row + step, y2, x2, d2);
    dot = LANES == 16 ? sum_of_16(dot) : sum_of_64(dot);
    if (WAVES > 1) {
      if ((t & 63) == 0) part[turn][t >> 6] = dot;
      __syncthreads();
      dot = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) dot += part[turn][w];
    }
    const float k = dot * over;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = 8 * (i * TEAM + t);
      float o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        o[j] = n * (g[i][j] * item(y[i], j) - item(x[i], j) * n * k);
        if (a.dh) o[j] += item(d[i], j);
      }
      store8((T*)a.dx + row * a.lddx + c, D - c, o);
    }
    if (AHEAD) {
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        y[i] = y2[i];
        x[i] = x2[i];
        d[i] = d2[i];
      }
    }
  }
  if (!a.dgamma) return;
  if (WAVES == 1) {                    // the teams' sums in order
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) sums[team][8 * (i * TEAM + t) + j] = acc[i][j];
    __syncthreads();
    for (int c = threadIdx.x; c < D; c += 256) {
      float sum = sums[0][c];
#pragma unroll
      for (int w = 1; w < TEAMS; ++w) sum += sums[w][c];
      partials[(int64_t)blockIdx.x * D + c] = sum;
    }
  } else {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = 8 * (i * TEAM + t);
      store8(partials + (int64_t)blockIdx.x * D + c, D - c, acc[i]);
    }
  }
}

// ---- backward, rows past 16384: the rows' products first, then the columns --------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void rmsnorm_dots_kernel(const NormBackArgs a, float* dots) {
  __shared__ float part[4];
  const int64_t row = blockIdx.x;
  const T *dy = (const T*)a.dy + row * a.lddy, *h = (const T*)a.h + row * a.ldh;
  const float n = a.rstd[row];
  float dot = 0.0f;
  for (int c = threadIdx.x; 8 * c < a.dim; c += 256) {
    float y[8], x[8], g[8];
    load8(dy + 8 * c, a.dim - 8 * c, y);
    load8(h + 8 * c, a.dim - 8 * c, x);
    if (a.gamma) load8(a.gamma + 8 * c, a.dim - 8 * c, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) dot += (a.gamma ? g[j] : 1.0f) * y[j] * (x[j] * n);
  }
  dot = sum_of_64(dot);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = dot;
  __syncthreads();
  if (threadIdx.x == 0) dots[row] = ((part[0] + part[1]) + (part[2] + part[3])) / (float)a.dim;
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
      acc[j] += y[j] * (x[j] * n);
      d[j] += n * (g[j] * y[j] - x[j] * n * k);
    }
    store8((T*)a.dx + row * a.lddx + c, left, d);
  }
  if (a.dgamma) store8(partials + (int64_t)blockIdx.y * a.dim + c, left, acc);
}

// Partial sums of gamma's gradient: workgroups of the one-pass kernel, or strands of rows.  As many as hide the loads, but every one is a row for
// sum_rows_kernel.  Both kernels, bf16, us: 100000 x 128 19.6 with 512, 22.2 with 256, 20.8 with 1024; 8192 x 300 12.3 with 1024, 13.0 with 512; 8192 x 1024 15.8 with 512, 18.4 with 1024; 5000 x 1500 25.2 with 512, 22.1 with 768,
// 8192 x 2048 27.7, 26.2, 27.7 with 1024, but 1000 x 1500 10.6, 12.2; 4096 x 4096 27.4 with 512, 31.9 with 256, 29.4 with 768; 4096 x 8192 52.0 with 256, 50.4 with 512,
// but 1000 x 16384 31.0, 37.5.
int backward_groups(int rows, int dim) {
  const int teams = dim <= 256 ? (rows + 15) / 16 : dim <= 1024 ? (rows + 3) / 4 : rows;
  const int most = dim <= 256 ? 512 : dim <= 512 ? 1024 : dim > 4096 ? 256 : dim > 1024 && dim <= 2048 && rows >= 4096 ? 768 : 512;
  return teams < most ? teams : most;
}

template <typename T>
hipError_t rmsnorm_backward_of(const NormBackArgs& a, hipStream_t s) {
  const int groups = backward_groups(a.rows, a.dim);
  const bool alone = groups == 1 && a.dim <= kOnePass;          // its sums are the gradient
  float* partials = alone ? a.dgamma : a.work;
  if (a.dim <= 128) rmsnorm_backward_kernel<T, 1, 1, true, 16><<<groups, 256, 0, s>>>(a, partials);
  else if (a.dim <= 256) rmsnorm_backward_kernel<T, 1, 2, true, 16><<<groups, 256, 0, s>>>(a, partials);
  else if (a.dim <= 512) rmsnorm_backward_kernel<T, 1, 1, true><<<groups, 256, 0, s>>>(a, partials);
  else if (a.dim <= 1024) rmsnorm_backward_kernel<T, 1, 2, true><<<groups, 256, 0, s>>>(a, partials);
  else if (a.dim <= 2048) rmsnorm_backward_kernel<T, 4, 1, true><<<groups, 256, 0, s>>>(a, partials);
  else if (a.dim <= 4096) rmsnorm_backward_kernel<T, 4, 2, true><<<groups, 256, 0, s>>>(a, partials);
  else if (a.dim <= 8192) rmsnorm_backward_kernel<T, 8, 2, true><<<groups, 512, 0, s>>>(a, partials);
  else if (a.dim <= kOnePass) rmsnorm_backward_kernel<T, 16, 2, false><<<groups, 1024, 0, s>>>(a, partials);
  else {
    float* dots = a.work;
    partials = a.work + (a.rows + 3) / 4 * 4;
    rmsnorm_dots_kernel<T><<<a.rows, 256, 0, s>>>(a, dots);
    rmsnorm_columns_kernel<T><<<dim3((a.dim + 2047) / 2048, groups), 256, 0, s>>>(a, dots, partials);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.dgamma || alone) return e;
  return launch_sum_rows(partials, groups, a.dim, a.dgamma, s);
}

// 32 columns (a line) and 32 strands of rows a workgroup.
__global__ __launch_bounds__(1024) void sum_rows_kernel(const float* __restrict__ in, int n, int cols, float* __restrict__ out) {
  __shared__ float part[32][33];
  const int lane = threadIdx.x & 31, strand = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float sum = 0.0f;
  if (c < cols) {
#pragma unroll 8
    for (int i = strand; i < n; i += 32) sum += in[(int64_t)i * cols + c];
  }
  part[strand][lane] = sum;
  __syncthreads();
  // strand s of column c: lane s of the 32 that add column c up
  sum = part[lane][strand];
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 32);
  if (lane == 0 && blockIdx.x * 32 + strand < cols) out[blockIdx.x * 32 + strand] = sum;
}

}  // namespace

hipError_t launch_sum_rows(const float* in, int n, int cols, float* out, hipStream_t s) {
  sum_rows_kernel<<<(cols + 31) / 32, 1024, 0, s>>>(in, n, cols, out);
  return hipGetLastError();
}

hipError_t launch_rmsnorm(int dtype, const NormArgs& a, hipStream_t s) { return dtype == 1 ? rmsnorm_of<bf16>(a, s) : rmsnorm_of<float>(a, s); }

size_t rmsnorm_backward_floats(int rows, int dim) {
  const size_t sums = (size_t)backward_groups(rows, dim) * dim;
  return dim > kOnePass ? (size_t)((rows + 3) / 4 * 4) + sums : sums > (size_t)dim ? sums : 0;
}

hipError_t launch_rmsnorm_backward(int dtype, const NormBackArgs& a, hipStream_t s) {
  return dtype == 1 ? rmsnorm_backward_of<bf16>(a, s) : rmsnorm_backward_of<float>(a, s);
}

}  // namespace slp
