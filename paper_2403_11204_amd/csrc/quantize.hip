// Matrices to 8 bits: e4m3 values and power-of-two scales, one for each 128 elements of a row or for each 128 x 128 block, row-major,
// transposed or both from one reading of the matrix; of a gradient, with the ReLU's mask applied first and the sums of the columns (the
// bias's gradient) taken along.
#include "eightbit_device.h"

namespace slp {
namespace {

// The steps on 8 elements of a row, two bf16 elements an instruction where there is one for it.  Magnitudes are compared as integers, which order like
// the values; kMags registers hold those of the columns.
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
template <typename T> constexpr int kMags = sizeof(T) == 2 ? 4 : 8;
__device__ __forceinline__ uint32_t word(const Raw<bf16>& v, int i) { return __builtin_bit_cast(u32x4, v.v)[i]; }
__device__ __forceinline__ u16x2 halves(uint32_t w) { return __builtin_bit_cast(u16x2, w); }
__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b) { return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(halves(a), halves(b))); }

// zero where m is not > 0
__device__ __forceinline__ void keep_positive(Raw<bf16>& v, const Raw<bf16>& m) {
  u32x4 o;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // as integers the positive values and infinity are 1 .. 0x7F80: all ones where 0x7F80 - (m - 1), stopped at zero, is not zero
    u16x2 d = __builtin_elementwise_sub_sat(u16x2{0x7F80, 0x7F80}, halves(word(m, i)) - u16x2{1, 1});
    d = u16x2{0, 0} - __builtin_elementwise_min(d, u16x2{1, 1});
    o[i] = word(v, i) & __builtin_bit_cast(uint32_t, d);
  }
  v.v = __builtin_bit_cast(bf16x8, o);
}
__device__ __forceinline__ void keep_positive(Raw<float>& v, const Raw<float>& m) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (!(m.v[j / 4][j % 4] > 0.0f)) v.v[j / 4][j % 4] = 0.0f;
}
// largest magnitude of the 8 elements; columns' raised to theirs
__device__ __forceinline__ uint32_t magnitudes(const Raw<bf16>& v, uint32_t (&columns)[4]) {
  uint32_t all = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t m = word(v, i) & 0x7FFF7FFFu;
    columns[i] = max_halves(columns[i], m);
    all = max_halves(all, m);
  }
  return umax(all & 0xFFFF0000u, all << 16);
}
__device__ __forceinline__ uint32_t magnitudes(const Raw<float>& v, uint32_t (&columns)[8]) {
  uint32_t all = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t m = magnitude(item(v, j));
    columns[j] = umax(columns[j], m);
    all = umax(all, m);
  }
  return all;
}
__device__ __forceinline__ uint32_t column(const uint32_t (&columns)[4], int j) { return j & 1 ? columns[j / 2] & 0xFFFF0000u : columns[j / 2] << 16; }
__device__ __forceinline__ uint32_t column(const uint32_t (&columns)[8], int j) { return columns[j]; }
__device__ __forceinline__ u32x2 row_e4m3(const Raw<bf16>& v, float scale) {
  return u32x2{to_e4m3(word(v, 0), word(v, 1), scale), to_e4m3(word(v, 2), word(v, 3), scale)};
}
__device__ __forceinline__ u32x2 row_e4m3(const Raw<float>& v, float scale) {
  return u32x2{to_e4m3(v.v[0][0], v.v[0][1], v.v[0][2], v.v[0][3], scale), to_e4m3(v.v[1][0], v.v[1][1], v.v[1][2], v.v[1][3], scale)};
}
// element j of four rows
__device__ __forceinline__ uint32_t column_e4m3(const Raw<bf16> (&v)[4], int j, float scale) {
  const uint32_t pick = j & 1 ? 0x07060302u : 0x05040100u;          // the high or the low half of both words
  return to_e4m3(__builtin_amdgcn_perm(word(v[1], j / 2), word(v[0], j / 2), pick), __builtin_amdgcn_perm(word(v[3], j / 2), word(v[2], j / 2), pick), scale);
}
__device__ __forceinline__ uint32_t column_e4m3(const Raw<float> (&v)[4], int j, float scale) {
  return to_e4m3(item(v[0], j), item(v[1], j), item(v[2], j), item(v[3], j), scale);
}

// Row-major alone, a scale for each 128 elements of a row: a chunk of 8 elements a lane, 16 lanes a scale, a workgroup 16 scales.  Bound by memory: 8192 x
// 8192 float32 58 us (338 MB, 5.8 TB/s), 8192 x 16384 bf16 72 us (404 MB, 5.6 TB/s); the tiles below take 77 for its
// transposed form.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const QuantizeArgs a) {
  const uint32_t blocks = (a.cols + 127) / 128, at = blockIdx.x * 16 + (threadIdx.x >> 4);       // (a matrix has fewer than 2^28 scales)
  const int64_t row = at / blocks;
  const int b = at % blocks, c = b * 128 + (threadIdx.x & 15) * 8, left = a.cols - c;
  if (row >= a.rows) return;           // (16 lanes together)
  Raw<T> v;
  fetch8((const T*)a.x + row * a.ldx + c, left, v);
  if (a.mask) {
    Raw<T> m;
    fetch8((const T*)a.mask + row * a.ldmask + c, left, m);
    keep_positive(v, m);
  }
  uint32_t columns[kMags<T>] = {};
  const uint32_t scale = scale_of(max_of_16(magnitudes(v, columns)));
  if (c < ((a.cols + 15) & ~15)) *(u32x2*)(a.q + row * a.ldq + c) = row_e4m3(v, scale_value(scale));
  if ((threadIdx.x & 15) == 0) a.scales[row * a.lds + b] = (uint8_t)scale;
}

// Everything else, a 128 x 128 tile a workgroup of 8 wavefronts: a thread holds 4 rows of 8 columns.  The transposed bytes go through LDS, a row
// of 128 bytes for each column of the tile; the 16-byte piece p of column c sits at p ^ (c / 8 mod 8), so that the lanes of a wavefront, which
// write 16 columns 8 apart, spread over the banks.  8 wavefronts: with 4, which hold twice as much each, a 4096 x 8192 bf16 gradient took 73 us, not 57.
// Bound by memory where there are many tiles, to both layouts: 8192 x 8192 float32 75 us (405 MB, 5.4 TB/s) with either kind of blocks.  4096 x 8192 bf16
// with a mask and sums (203 MB) takes 33 us in repeated calls, whose inputs the last cache holds, but 47 to 56 behind other work (3.6 to 4.3 TB/s): a workgroup loads, exchanges
// and stores its one tile in turns.  By the steps of one tile, 1.5 us behind the 2.5 of an empty launch, where there are few.
template <typename T, int BLOCK>
__global__ __launch_bounds__(512) void quantize_tile_kernel(const QuantizeArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t turned[128 * 128];
  __shared__ __attribute__((aligned(16))) uint32_t cmax[8][128];
  __shared__ __attribute__((aligned(16))) float csum[8][128];
  const int t = threadIdx.x, wave = t >> 6, g = t >> 4, cc = t & 15;
  const int tilesM = (a.rows + 127) / 128, tilesN = (a.cols + 127) / 128;
  const int64_t tm = blockIdx.x / tilesN;
  const int tn = blockIdx.x % tilesN;
  const int64_t m0 = tm * 128;
  const int c0 = tn * 128 + cc * 8, left = a.cols - c0;
  Raw<T> v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t row = m0 + 4 * g + i;
    fetch8((const T*)a.x + row * a.ldx + c0, row < a.rows ? left : 0, v[i]);
  }
  if (a.mask) {
    Raw<T> m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t row = m0 + 4 * g + i;
      fetch8((const T*)a.mask + row * a.ldmask + c0, row < a.rows ? left : 0, m[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) keep_positive(v[i], m[i]);
  }
  // largest magnitudes: of the rows (16 lanes each), of the columns (a thread's 4 rows, 4 lanes of a wavefront, 8 wavefronts)
  uint32_t rmax[4], columns[kMags<T>] = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) rmax[i] = magnitudes(v[i], columns);
  if (BLOCK == 128 || a.qt) {
    u32x4 k[2];
#pragma unroll
    for (int j = 0; j < 8; ++j) k[j / 4][j % 4] = max_of_rows(column(columns, j));
    if ((t & 63) < 16) {
      *(u32x4*)&cmax[wave][cc * 8] = k[0];
      *(u32x4*)&cmax[wave][cc * 8 + 4] = k[1];
    }
  }
  if (a.sums) {
    f32x4 sum[2];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j / 4][j % 4] = sum_of_rows((item(v[0], j) + item(v[1], j)) + (item(v[2], j) + item(v[3], j)));
    if ((t & 63) < 16) {
      *(f32x4*)&csum[wave][cc * 8] = sum[0];
      *(f32x4*)&csum[wave][cc * 8 + 4] = sum[1];
    }
  }
  __syncthreads();
  if (a.sums && t < 128 && tn * 128 + t < a.cols) {
    float sum = csum[0][t];
#pragma unroll
    for (int w = 1; w < 8; ++w) sum += csum[w][t];
    (tilesM == 1 ? a.sums : a.work + tm * a.cols)[tn * 128 + t] = sum;
  }
  // the columns' scales, a column a thread, in place of the first wavefront's largest magnitudes (every thread reading all eight took 1.6 us more)
  if (BLOCK == 1 && a.qt) {
    if (t < 128) {
      uint32_t k = cmax[0][t];
#pragma unroll
      for (int w = 1; w < 8; ++w) k = umax(k, cmax[w][t]);
      k = scale_of(k);
      if (tn * 128 + t < a.cols) a.scales_t[(int64_t)(tn * 128 + t) * a.ldst + tm] = (uint8_t)k;
      cmax[0][t] = k;
    }
    __syncthreads();
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
      if (row < a.rows) {
        if (c0 < ((a.cols + 15) & ~15)) *(u32x2*)(a.q + row * a.ldq + c0) = row_e4m3(v[i], scale_value(scale));
        if (BLOCK == 1 && cc == 0) a.scales[row * a.lds + tn] = (uint8_t)scale;
      }
    }
  }
  if (a.qt) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = cc * 8 + j;
      const uint32_t scale = BLOCK == 128 ? all : cmax[0][c];
      *(uint32_t*)(turned + c * 128 + (((g >> 2) ^ (cc & 7)) << 4) + (g & 3) * 4) = column_e4m3(v, j, scale_value(scale));
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
