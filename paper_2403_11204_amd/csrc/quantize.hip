// Matrices to 8 bits: e4m3 values and power-of-two scales, one for each 128 elements of a row or for each 128 x 128 block, row-major,
// transposed or both from one reading of the matrix; of a gradient, with the ReLU's mask applied first and the sums of the columns (the
// bias's gradient) taken along.
#include "eightbit_device.h"

namespace slp {
namespace {

// Row-major alone, a scale for each 128 elements of a row: a chunk of 8 elements a lane, 16 lanes a scale, a workgroup 16 scales.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const QuantizeArgs a) {
  const int blocks = (a.cols + 127) / 128;
  const int64_t at = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int64_t row = at / blocks;
  const int b = (int)(at % blocks), c = b * 128 + (threadIdx.x & 15) * 8, left = a.cols - c;
  if (row >= a.rows) return;           // (16 lanes together)
  float v[8];
  load8((const T*)a.x + row * a.ldx + c, left, v);
  if (a.mask) {
    float m[8];
    load8((const T*)a.mask + row * a.ldmask + c, left, m);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (!(m[j] > 0.0f)) v[j] = 0.0f;
  }
  uint32_t amax = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) amax = umax(amax, magnitude(v[j]));
  const uint32_t scale = scale_of(max_of_16(amax));
  const float up = inverse_scale(scale);
  if (c < ((a.cols + 15) & ~15))
    *(u32x2*)(a.q + row * a.ldq + c) = u32x2{to_e4m3(v[0] * up, v[1] * up, v[2] * up, v[3] * up), to_e4m3(v[4] * up, v[5] * up, v[6] * up, v[7] * up)};
  if ((threadIdx.x & 15) == 0) a.scales[row * a.lds + b] = (uint8_t)scale;
}

// Everything else, a 128 x 128 tile a workgroup of 8 wavefronts: a thread holds 4 rows of 8 columns.  The transposed bytes go through LDS, a row
// of 128 bytes for each column of the tile; the 16-byte piece p of column c sits at p ^ (c / 8 mod 8), so that the lanes of a wavefront, which
// write 16 columns 8 apart, spread over the banks.
template <typename T, int BLOCK>
__global__ __launch_bounds__(512) void quantize_tile_kernel(const QuantizeArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t turned[128 * 128];
  __shared__ uint32_t cmax[8][128];
  __shared__ float csum[8][128];
  const int t = threadIdx.x, wave = t >> 6, g = t >> 4, cc = t & 15;
  const int tilesM = (a.rows + 127) / 128, tilesN = (a.cols + 127) / 128;
  const int64_t tm = blockIdx.x / tilesN;
  const int tn = blockIdx.x % tilesN;
  const int64_t m0 = tm * 128;
  const int c0 = tn * 128 + cc * 8, left = a.cols - c0;
  float v[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t row = m0 + 4 * g + i;
    load8((const T*)a.x + row * a.ldx + c0, row < a.rows ? left : 0, v[i]);
  }
  if (a.mask) {
    float m[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t row = m0 + 4 * g + i;
      load8((const T*)a.mask + row * a.ldmask + c0, row < a.rows ? left : 0, m[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (!(m[i][j] > 0.0f)) v[i][j] = 0.0f;
  }
  // largest magnitudes: of the rows (16 lanes each), of the columns (a thread's 4 rows, 4 lanes of a wavefront, 8 wavefronts)
  uint32_t rmax[4] = {0, 0, 0, 0}, kmax[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float sum = 0.0f;
    kmax[j] = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t m = magnitude(v[i][j]);
      rmax[i] = umax(rmax[i], m);
      kmax[j] = umax(kmax[j], m);
      sum += v[i][j];
    }
    if (BLOCK == 128 || a.qt) {
      kmax[j] = max_of_rows(kmax[j]);
      if ((t & 63) < 16) cmax[wave][cc * 8 + j] = kmax[j];
    }
    if (a.sums) {
      sum = sum_of_rows(sum);
      if ((t & 63) < 16) csum[wave][cc * 8 + j] = sum;
    }
  }
  __syncthreads();
  if (a.sums && t < 128 && tn * 128 + t < a.cols) {
    float sum = csum[0][t];
#pragma unroll
    for (int w = 1; w < 8; ++w) sum += csum[w][t];
    (tilesM == 1 ? a.sums : a.work + tm * a.cols)[tn * 128 + t] = sum;
  }
  uint32_t all = 0;
  if (BLOCK == 128) {
#pragma unroll
    for (int w = 0; w < 8; ++w) all = umax(all, umax(cmax[w][t & 63], cmax[w][64 + (t & 63)]));
    all = scale_of(max_of_rows(max_of_16(all)));
    if (t == 0) {
      if (a.q) a.scales[tm * a.lds + tn] = (uint8_t)all;
      if (a.qt) a.scales_t[(int64_t)tn * a.ldst + tm] = (uint8_t)all;
    }
  }
  if (a.q) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t row = m0 + 4 * g + i;
      const uint32_t scale = BLOCK == 128 ? all : scale_of(max_of_16(rmax[i]));
      const float up = inverse_scale(scale);
      if (row < a.rows) {
        if (c0 < ((a.cols + 15) & ~15))
          *(u32x2*)(a.q + row * a.ldq + c0) = u32x2{to_e4m3(v[i][0] * up, v[i][1] * up, v[i][2] * up, v[i][3] * up),
                                                   to_e4m3(v[i][4] * up, v[i][5] * up, v[i][6] * up, v[i][7] * up)};
        if (BLOCK == 1 && cc == 0) a.scales[row * a.lds + tn] = (uint8_t)scale;
      }
    }
  }
  if (a.qt) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = cc * 8 + j;
      uint32_t scale = all;
      if (BLOCK == 1) {
        uint32_t k = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) k = umax(k, cmax[w][c]);
        scale = scale_of(k);
        if (g == 0 && c0 + j < a.cols) a.scales_t[(int64_t)(c0 + j) * a.ldst + tm] = (uint8_t)scale;
      }
      const float up = inverse_scale(scale);
      *(uint32_t*)(turned + c * 128 + (((g >> 2) ^ (cc & 7)) << 4) + (g & 3) * 4) = to_e4m3(v[0][j] * up, v[1][j] * up, v[2][j] * up, v[3][j] * up);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int c = i * 64 + (t >> 3), p = t & 7;
      if (tn * 128 + c < a.cols && m0 + 16 * p < a.rows)          // zeros up to the next 16 bytes
        *(u32x4*)(a.qt + (int64_t)(tn * 128 + c) * a.ldqt + m0 + 16 * p) = *(const u32x4*)(turned + c * 128 + ((p ^ ((c >> 3) & 7)) << 4));
    }
  }
}

int64_t tile_count(const QuantizeArgs& a) { return (int64_t)((a.rows + 127) / 128) * ((a.cols + 127) / 128); }

template <typename T>
hipError_t quantize_of(const QuantizeArgs& a, hipStream_t s) {
  if (!a.qt && !a.sums && a.block == 1) {
    const int64_t scales = (int64_t)a.rows * ((a.cols + 127) / 128);
    quantize_rows_kernel<T><<<(unsigned)((scales + 15) / 16), 256, 0, s>>>(a);
    return hipGetLastError();
  }
  const unsigned tiles = (unsigned)tile_count(a);
  if (a.block == 128) quantize_tile_kernel<T, 128><<<tiles, 512, 0, s>>>(a);
  else quantize_tile_kernel<T, 1><<<tiles, 512, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.sums || a.rows <= 128) return e;      // (a single tile's height has stored its sums itself)
  return launch_sum_rows(a.work, (a.rows + 127) / 128, a.cols, a.sums, s);
}

}  // namespace

size_t quantize_floats(int rows, int cols) { return rows <= 128 ? 0 : (size_t)((rows + 127) / 128) * cols; }

hipError_t launch_quantize(int dtype, const QuantizeArgs& a, hipStream_t s) { return dtype == 1 ? quantize_of<bf16>(a, s) : quantize_of<float>(a, s); }

}  // namespace slp
