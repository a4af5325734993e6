// The norm of many tensors together and their scaling to a given norm.
//
//   norm = sqrt(sum over all tensors of sum(g^2));  g <- c g, c = min(1, max_norm / (norm + 1e-6))
//
// Squares and their sums are float64, in which no float32 value's square overflows or underflows; every workgroup adds up its own elements
// in a fixed order and stores one partial sum, and whoever needs the total adds up all partial sums in the same order: no atomics, the same
// bits every time.  A norm that is not finite in float32, as the caller sees it, leaves the gradients as they are (c = 1): it is the caller's to skip the update.
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

// f(tensor, its chunk) for each chunk of this workgroup.  Chunks are dealt out in turns, to one workgroup for each compute unit, so that all of
// them read and write within 8 MB at a time: 549 million float32 values, norm / clipping 334 / 1141 us (6.5 TB/s / 5.8 for 6.6 GB) against 349 / 1172
// with two workgroups each and 375 / 1201 with four; 455 / 1357 with chunks of 16 KB, 355 / 1187 with 64 KB.  These are repeated calls; behind other work the squares take 371, between
// two clippings 386 (5.7 TB/s).
template <typename F>
__device__ __forceinline__ void each_chunk(const ClipTable& t, F f) {
  int i = 0;
  for (int c = blockIdx.x; c < t.chunk0[t.n]; c += gridDim.x) {
    if (c >= t.chunk0[i + 1]) {        // the last tensor that starts there or before: 6 steps, where one by one 48 tensors took 1 us more a launch
#pragma unroll
      for (int step = 32; step > 0; step >>= 1)
        if (i + step < t.n && t.chunk0[i + step] <= c) i += step;
    }
    f(i, c - t.chunk0[i]);
  }
}

// Chunk c of a tensor: a thread's elements of it, 8 at a time, all loads under way together; f(first of 8, how many of them exist, they).
template <typename T, typename F>
__device__ __forceinline__ void each_eight(const T* p, int64_t count, int c, F f) {
  constexpr int kElements = kClipChunk / (int)sizeof(T), kVectors = kElements / (256 * 8);
  const int64_t first = (int64_t)c * kElements, left = count - first;
  const int n = left < kElements ? (int)left : kElements;
  Raw<T> v[kVectors];
#pragma unroll
  for (int i = 0; i < kVectors; ++i) {
    const int k = (i * 256 + threadIdx.x) * 8;
    fetch8(p + first + k, n - k, v[i]);
  }
#pragma unroll
  for (int i = 0; i < kVectors; ++i) {
    const int k = (i * 256 + threadIdx.x) * 8;
    f(first + k, n - k, v[i]);
  }
}

template <typename T>
__device__ __forceinline__ double squares(const T* p, int64_t count, int c) {
  double sum = 0.0;
  each_eight(p, count, c, [&](int64_t, int, const Raw<T>& v) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const double x = (double)item(v, j);
      sum += x * x;
    }
  });
  return sum;
}

__global__ __launch_bounds__(256) void square_sums_kernel(const ClipTable t, double* __restrict__ partials) {
  double sum = 0.0;
  each_chunk(t, [&](int i, int c) {
    if ((t.bf16 >> i) & 1) sum += squares((const bf16*)t.in[i], t.count[i], c);
    else sum += squares((const float*)t.in[i], t.count[i], c);
  });
  sum = sum_of_256(sum);
  if (threadIdx.x == 0) partials[blockIdx.x] = sum;
}

__global__ __launch_bounds__(256) void norm_of_kernel(const double* __restrict__ partials, int n, float* __restrict__ norm) {
  const double x = total(partials, n);
  if (threadIdx.x == 0) *norm = (float)sqrt(x);
}

// The factor as m 2^e, m in [0.5, 1]: it may lie below float32's range where the values scaled by it do not.
template <typename T>
__device__ __forceinline__ void scaled(const T* in, T* out, int64_t count, int c, float m, int e) {
  each_eight(in, count, c, [&](int64_t k, int n, const Raw<T>& v) {
    float o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = ldexpf(item(v, j) * m, e);
    store8(out + k, n, o);
  });
}

__global__ __launch_bounds__(256) void scale_kernel(const ClipTable t, const double* __restrict__ partials, int n, float max_norm, float* __restrict__ norm) {
  const double x = sqrt(total(partials, n));
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)x;
  const double ratio = (double)max_norm / (x + 1e-6);
  int e = 0;
  const float m = (float)x < INFINITY && ratio < 1.0 ? (float)frexp(ratio, &e) : 1.0f;
  each_chunk(t, [&](int i, int c) {
    if (m == 1.0f && e == 0 && t.in[i] == t.out[i]) return;
    if ((t.bf16 >> i) & 1) scaled((const bf16*)t.in[i], (bf16*)t.out[i], t.count[i], c, m, e);
    else scaled((const float*)t.in[i], (float*)t.out[i], t.count[i], c, m, e);
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
