// The norm of many tensors together and their scaling to a given norm.
//
//   norm = sqrt(sum over all tensors of sum(g^2));  g <- c g, c = min(1, max_norm / (norm + 1e-6))
//
// Squares and their sums are float64, in which no float32 value's square overflows or underflows; every workgroup adds up its own elements
// in a fixed order and stores one partial sum, and whoever needs the total adds up all partial sums in the same order: no atomics, the same
// bits every time.  A norm that is not finite leaves the gradients as they are (c = 1): it is the caller's to see and to skip the update.
#include "eightbit_device.h"

namespace slp {
namespace {

__device__ __forceinline__ double sum_of_256(double x) {
  __shared__ double part[4];
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
  __syncthreads();                     // (an earlier call's reads)
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

// The sum of all partial sums, in every thread of the workgroup.
__device__ __forceinline__ double total(const double* __restrict__ partials, int n) {
  double x = 0.0;
  for (int i = threadIdx.x; i < n; i += 256) x += partials[i];
  return sum_of_256(x);
}

// f(tensor, first element, elements) for each chunk of this workgroup: chunks are dealt out in turns.
template <typename F>
__device__ __forceinline__ void each_chunk(const ClipTable& t, F f) {
  int i = 0;
  for (int c = blockIdx.x; c < t.chunk0[t.n]; c += gridDim.x) {
    while (c >= t.chunk0[i + 1]) ++i;
    const int64_t first = (int64_t)(c - t.chunk0[i]) * kClipChunk, left = t.count[i] - first;
    f(i, first, (int)(left < kClipChunk ? left : kClipChunk));
  }
}

template <typename T>
__device__ __forceinline__ double squares(const T* p, int n) {
  double sum = 0.0;
  for (int k = threadIdx.x * 8; k < n; k += 256 * 8) {
    float v[8];
    load8(p + k, n - k, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += (double)v[j] * (double)v[j];
  }
  return sum;
}

__global__ __launch_bounds__(256) void square_sums_kernel(const ClipTable t, double* __restrict__ partials) {
  double sum = 0.0;
  each_chunk(t, [&](int i, int64_t first, int n) {
    if ((t.bf16 >> i) & 1) sum += squares((const bf16*)t.in[i] + first, n);
    else sum += squares((const float*)t.in[i] + first, n);
  });
  sum = sum_of_256(sum);
  if (threadIdx.x == 0) partials[blockIdx.x] = sum;
}

__global__ __launch_bounds__(256) void norm_of_kernel(const double* __restrict__ partials, int n, float* __restrict__ norm) {
  const double x = total(partials, n);
  if (threadIdx.x == 0) *norm = (float)sqrt(x);
}

template <typename T>
__device__ __forceinline__ void scaled(const T* in, T* out, int n, float c) {
  for (int k = threadIdx.x * 8; k < n; k += 256 * 8) {
    float v[8];
    load8(in + k, n - k, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= c;
    store8(out + k, n - k, v);
  }
}

__global__ __launch_bounds__(256) void scale_kernel(const ClipTable t, const double* __restrict__ partials, int n, float max_norm, float* __restrict__ norm) {
  const double x = sqrt(total(partials, n));
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)x;
  const double ratio = (double)max_norm / (x + 1e-6);
  const float c = x < INFINITY && ratio < 1.0 ? (float)ratio : 1.0f;
  each_chunk(t, [&](int i, int64_t first, int n) {
    if (c == 1.0f && t.in[i] == t.out[i]) return;
    if ((t.bf16 >> i) & 1) scaled((const bf16*)t.in[i] + first, (bf16*)t.out[i] + first, n, c);
    else scaled((const float*)t.in[i] + first, (float*)t.out[i] + first, n, c);
  });
}

}  // namespace

hipError_t launch_square_sums(const ClipTable& t, int groups, double* partials, hipStream_t s) {
  square_sums_kernel<<<groups, 256, 0, s>>>(t, partials);
  return hipGetLastError();
}

hipError_t launch_norm_of(const double* partials, int n, float* norm, hipStream_t s) {
  norm_of_kernel<<<1, 256, 0, s>>>(partials, n, norm);
  return hipGetLastError();
}

hipError_t launch_scale(const ClipTable& t, int groups, const double* partials, int n, float max_norm, float* norm, hipStream_t s) {
  scale_kernel<<<groups, 256, 0, s>>>(t, partials, n, max_norm, norm);
  return hipGetLastError();
}

}  // namespace slp
