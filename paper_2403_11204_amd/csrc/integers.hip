// 8-bit integers with a scale for each row (a token of the activations, an output channel of the weights):
//
//   q = round(127 x / max|x|), scale = max|x| / 127;   out[m][n] = act(sa[m] sb[n] sum over k of a[m][k] b[n][k] + bias[n])
//
// The sums are integers, exact whatever the order: contractions of up to 131071 stay below 2^31.  v_mfma_i32_16x16x64_i8 does 64 k of a 16 x 16 block in 16
// cycles, as much as the 8-bit floating-point forms.  Operands are laid out, loaded and passed (in the order B, A: a lane holds 4 consecutive columns of one
// row of the output) as in product.hip; with nothing to convert and no scales on the way, a k-tile is reads and matrix instructions only.
#include "eightbit_device.h"
#include "gemm_launch.h"
#include "long_tile.h"
#include "product_shapes.h"

namespace slp {
namespace {

constexpr int kXcds = 8;
constexpr uint32_t kOutOfRange = 0x80000000u;     // byte offset past the end of every tile

// ---- quantising -----------------------------------------------------------------------------------
// The integer nearest to 127 x / amax, ties to even, of the real quotient: x times a reciprocal is 2^-23 of it off at most, 1.6e-5, and where it lies that near
// to a half the quotient is taken in 64 bits (its distance from a half is then 2^-34 or nothing).
__device__ __forceinline__ int nearest(float x, float inverse, float amax) {
  const float t = x * inverse, r = __builtin_rintf(t);
  if (fabsf(fabsf(t - r) - 0.5f) < 4e-5f) return (int)__builtin_rint(127.0 * (double)x / (double)amax);
  return (int)r;
}
__device__ __forceinline__ u32x2 nearest8(const float (&v)[8], float inverse, float amax) {
  u32x2 o = {0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e / 4] |= (uint32_t)(nearest(v[e], inverse, amax) & 255) << (8 * (e % 4));
  return o;
}

// A row on LANES threads (16, a wavefront or the workgroup), NV vectors of 8 elements each, held in registers between the two uses; LONG: read again, any
// length.  Bound by memory: one reading, one writing of a byte for each element; 8192 x 16384 bf16 89 us (4.5 TB/s), 1 x 4096 2.5, a launch.
template <typename T, int LANES, int NV, bool LONG>
__global__ __launch_bounds__(256) void quantize_integers_kernel(const IntegersArgs a) {
  __shared__ uint32_t most[4];
  constexpr int TEAMS = 256 / LANES;
  const int t = threadIdx.x, l = t % LANES;
  const int64_t row = (int64_t)blockIdx.x * TEAMS + t / LANES;
  const bool in = row < a.rows;
  const T* const x = (const T*)a.x + (in ? row : 0) * a.ldx;
  float v[NV][8];
  uint32_t amax = 0;
  if constexpr (LONG) {
    for (int c = l * 8; c < a.cols; c += LANES * 8) {
      load8(x + c, a.cols - c, v[0]);
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = umax(amax, magnitude(v[0][e]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) load8(x + (l + i * LANES) * 8, in ? a.cols - (l + i * LANES) * 8 : 0, v[i]);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = umax(amax, magnitude(v[i][e]));
  }
  amax = max_of_16(amax);
  if constexpr (LANES > 16) amax = max_of_rows(amax);
  if constexpr (LANES > 64) {
    if ((t & 63) == 0) most[t >> 6] = amax;
    __syncthreads();
    amax = umax(umax(most[0], most[1]), umax(most[2], most[3]));
  }
  if (!in) return;
  // an infinity or a NaN: a scale that is NaN; below 2^-100 the quotient of values 2^64 times as large, where 127 / amax is finite
  const bool number = amax < 0x7F800000u && amax != 0;
  float m = __builtin_bit_cast(float, amax);
  const float up = m < 7.8886e-31f ? 18446744073709551616.0f : 1.0f;
  if (l == 0) a.scales[row] = amax >= 0x7F800000u ? NAN : m / 127.0f;
  m *= up;
  const float inverse = number ? 127.0f / m : 0.0f;
  int8_t* const q = a.q + row * a.ldq;
  const int end = (a.cols + 15) & ~15;
  auto put = [&](int c, float (&w)[8]) {
    if (c >= end) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = number ? w[e] * up : 0.0f;
    *(u32x2*)(q + c) = nearest8(w, inverse, number ? m : 1.0f);
  };
  if constexpr (LONG) {
    for (int c = l * 8; c < end; c += LANES * 8) {
      load8(x + c, a.cols - c, v[0]);
      put(c, v[0]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) put((l + i * LANES) * 8, v[i]);
  }
}

// ---- products -------------------------------------------------------------------------------------
__device__ __forceinline__ i32x4 mfma(const u32x4& b, const u32x4& a, const i32x4& acc) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, b), __builtin_bit_cast(i32x4, a), acc, 0, 0, 0);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_of(const void* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00020000);
}

// Scales and bias of 4 consecutive columns; what is past their end is the last one's, for columns that nobody stores.
struct Columns {
  f32x4 scale, bias;
};
__device__ __forceinline__ Columns columns_at(const IntegerProductArgs& g, int n) {
  Columns c;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int at = n + e < g.N ? n + e : g.N - 1;
    c.scale[e] = g.sb[at];
    c.bias[e] = g.bias ? g.bias[at] : 0.0f;
  }
  return c;
}
__device__ __forceinline__ float row_scale(const IntegerProductArgs& g, int m) { return g.sa[m < g.M ? m : g.M - 1]; }
// A row's largest value may be anything up to 3e38, and the sum (below 2^31) times its scale beyond float32's range where the result is not: for rows from 2^96 on (LARGE: a wavefront has
// one) the column's scale comes first, which leaves the range only where the result does, too.  Nothing is lost at the other end: the sum is an integer, and that times a number below 2^-126
// is exact.  (3000 x 3000 x 304 in bf16 17.0 us without any of this, 17.3 with a branch around a wavefront's whole tail, 19.1 with one in
// each block, 18.6 with exponents put together by ldexp; smaller tiles and longer contractions are equal.)
__device__ __forceinline__ bool is_large(float scale) { return fabsf(scale) >= 7.9228163e28f; }
template <bool LARGE>
__device__ __forceinline__ f32x4 finished(const IntegerProductArgs& g, const i32x4& sum, float scale, const Columns& c) {
  const float least = g.relu ? 0.0f : -INFINITY;
  const bool swap = LARGE && is_large(scale);
  f32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float first = swap ? c.scale[e] : scale, second = swap ? scale : c.scale[e];
    v[e] = __builtin_elementwise_maximum(__builtin_fmaf((float)sum[e] * first, second, c.bias[e]), least);       // (a NaN stays one)
  }
  return v;
}
// tail(LARGE) for a wavefront whose lanes hold N rows' scales each
template <int N, typename F>
__device__ __forceinline__ void with_scales(const float (&scale)[N], F tail) {
  bool large = false;
#pragma unroll
  for (int i = 0; i < N; ++i) large |= is_large(scale[i]);
  if (__builtin_amdgcn_ballot_w64(large)) tail(std::true_type{});
  else tail(std::false_type{});
}
// Four consecutive columns n .. n + 3 of row m.
__device__ __forceinline__ void store4(const IntegerProductArgs& g, int m, int n, f32x4 v) {
  if (m >= g.M || n >= g.N) return;
  const int64_t at = (int64_t)m * g.ldo + n;
  const int left = g.N - n;
  if (g.out_dtype == 1) {
    bf16* out = (bf16*)g.out + at;
    const bf16x4 o = {(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
    if (left >= 4) ((AnyBf16x4*)out)->v = o;
    else
      for (int e = 0; e < left; ++e) out[e] = o[e];
  } else {
    float* out = (float*)g.out + at;
    if (left >= 4) ((AnyF32x4*)out)->v = v;
    else
      for (int e = 0; e < left; ++e) out[e] = v[e];
  }
}

// BM x BN tile, 4 wavefronts in a 2 x 2 grid, NS LDS stages of a k-tile of 128 each, one barrier a k-tile.  NG such groups of wavefronts
// take a part of the contraction each (kper k-tiles) and are added up at the end.  blockIdx.y: part of the contraction of a whole workgroup; several parts
// leave partial sums for integer_join_kernel.  48 x 4096 x 8192 10.7 us (3.1 TB/s of B, 2.5 of them the launch), 1000 x 3001 x 1500 float32 13.8: three workgroups a
// compute unit, loads, barriers and LDS in turn, 12 MB of output.
template <int BM, int BN, int NS, int NG>
__global__ __launch_bounds__(256 * NG) void integer_tile_kernel(const IntegerProductArgs g, int kper) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ __attribute__((aligned(16))) unsigned char all_smem[];
  constexpr int A_BYTES = BM * 128, STAGE = (BM + BN) * 128;
  const int group = NG > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) : 0;
  unsigned char* const smem = all_smem + group * (NS * STAGE);
  constexpr int LA = BM / 32, LB = BN / 32, NLD = LA + LB;                               // loads a lane per k-tile
  constexpr int MI = BM / 32, NI = BN / 32;
  const int tilesM = (g.M + BM - 1) / BM, tilesN = (g.N + BN - 1) / BN, total = tilesM * tilesN;
  int tid;
  {
    const int pid = blockIdx.x, xcd = pid % kXcds, q = pid / kXcds, base = total / kXcds, rem = total % kXcds;
    tid = xcd * base + (xcd < rem ? xcd : rem) + q;
  }
  constexpr int kGroup = 8;
  const int width = kGroup * tilesN, first = tid / width * kGroup, rows = tilesM - first < kGroup ? tilesM - first : kGroup;
  const int m0 = (first + tid % width % rows) * BM, n0 = tid % width / rows * BN;
  const int t = threadIdx.x & 255, lane = t & 63, w = t >> 6, wm = w & 1, wn = w >> 1, lgrp = lane >> 4, lrow = lane & 15;

  const int nk = (g.K + 127) / 128, Kr = (g.K + 15) & ~15;
  const int k0 = (blockIdx.y * NG + group) * kper, k1 = k0 + kper < nk ? k0 + kper : nk;
  const int ra = g.M - m0 < BM ? g.M - m0 : BM, rb = g.N - n0 < BN ? g.N - n0 : BN;        // rows of the tile that exist
  const __amdgpu_buffer_rsrc_t rsrcA = rsrc_of(g.a + (int64_t)m0 * g.lda, (ra - 1) * g.lda + Kr);
  const __amdgpu_buffer_rsrc_t rsrcB = rsrc_of(g.b + (int64_t)n0 * g.ldb, (rb - 1) * g.ldb + Kr);
  // a load of the workgroup fills 32 rows, lane l of wavefront w the 16-byte piece l % 8 of row 8 w + l / 8; piece c of a row is chunk
  // c ^ (row / 2 mod 8), which spreads the 16 rows of a fragment over all LDS banks
  const int prow = w * 8 + (lane >> 3), chunk = (lane & 7) ^ ((prow >> 1) & 7);
  uint32_t voff[LA + LB];
#pragma unroll
  for (int i = 0; i < LA; ++i) voff[i] = prow + 32 * i < ra ? (uint32_t)((prow + 32 * i) * g.lda + chunk * 16) : kOutOfRange;
#pragma unroll
  for (int i = 0; i < LB; ++i) voff[LA + i] = prow + 32 * i < rb ? (uint32_t)((prow + 32 * i) * g.ldb + chunk * 16) : kOutOfRange;
  typedef __attribute__((address_space(3))) void* lds_ptr_t;
  const int lds_wave = __builtin_amdgcn_readfirstlane(w * 1024);
  auto load = [&](int kt, int stage) {
    unsigned char* const st = smem + stage * STAGE;
    const bool in = kt < k1 && kt * 128 + chunk * 16 < Kr;
    const uint32_t koff = (uint32_t)kt * 128u;
#pragma unroll
    for (int i = 0; i < LA + LB; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(i < LA ? rsrcA : rsrcB, (lds_ptr_t)(st + lds_wave + i * 4096), 16,
                                               in && voff[i] != kOutOfRange ? voff[i] + koff : kOutOfRange, 0, 0, 0);
  };
  const uint32_t fragA = (uint32_t)((wm * (BM / 2) + lrow) * 128), fragB = (uint32_t)(A_BYTES + (wn * (BN / 2) + lrow) * 128);
  const uint32_t x0 = (uint32_t)((lgrp ^ ((lane >> 1) & 7)) << 4), x1 = x0 ^ 64;

  i32x4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = i32x4{0, 0, 0, 0};

  // a k-tile that everybody's loads have filled
  auto multiply = [&](int kt, auto ragged) {
    const unsigned char* const st = smem + (kt - k0) % NS * STAGE;
    u32x4 a[MI][2], b[NI][2];
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      b[j][0] = *(const u32x4*)(st + fragB + j * 2048 + x0);
      b[j][1] = *(const u32x4*)(st + fragB + j * 2048 + x1);
      if constexpr (ragged) {
        b[j][0] &= first_bytes((g.K & 127) - 16 * lgrp);
        b[j][1] &= first_bytes((g.K & 127) - 64 - 16 * lgrp);
      }
    }
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      a[i][0] = *(const u32x4*)(st + fragA + i * 2048 + x0);
      a[i][1] = *(const u32x4*)(st + fragA + i * 2048 + x1);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = mfma(b[j][h], a[i][h], acc[i][j]);
  };
#pragma unroll
  for (int s = 0; s < NS - 1; ++s) load(k0 + s, s);
  // the last k-tile has a copy of its own behind the loop where it ends inside 16 bytes
  const int end = NG > 1 ? k0 + kper : k1, whole = (g.K & 15) && k0 < nk && end >= nk ? nk - 1 : end;
  for (int kt = k0; kt < whole; ++kt) {
    // this wavefront's part of k-tile kt has landed and its reads of the last one are done; behind the barrier, everybody's
    __builtin_amdgcn_s_waitcnt(SLP_VMCNT_LGKM0((NS - 2) * NLD));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    load(kt + NS - 1, (kt - k0 + NS - 1) % NS);
    if (NG > 1 && kt >= k1) continue;            // (a shorter part takes the others' barriers)
    multiply(kt, std::false_type{});
  }
  if (whole < end) {
    __builtin_amdgcn_s_waitcnt(SLP_VMCNT_LGKM0((NS - 2) * NLD));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    multiply(nk - 1, std::true_type{});
    for (int kt = nk; kt < end; ++kt) __builtin_amdgcn_s_barrier();
  }
  __builtin_amdgcn_s_waitcnt(SLP_VMCNT(0));      // no load into LDS may outlive the workgroup
  if constexpr (NG > 1) {
    // the other groups' sums, 16 bytes of each lane side by side
    __syncthreads();
    i32x4* const sums = (i32x4*)all_smem + t;
    if (group > 0) {
#pragma unroll
      for (int i = 0; i < MI * NI; ++i) sums[((group - 1) * MI * NI + i) * 256] = acc[i / NI][i % NI];
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int v = 0; v < NG - 1; ++v)
#pragma unroll
      for (int i = 0; i < MI * NI; ++i) acc[i / NI][i % NI] += sums[(v * MI * NI + i) * 256];
  }
  if (gridDim.y > 1) {
    const int64_t ldp = (g.N + 3) & ~3;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int n = n0 + wn * (BN / 2) + j * 16 + 4 * lgrp;
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const int m = m0 + wm * (BM / 2) + i * 16 + lrow;
        if (m < g.M && n < g.N) *(i32x4*)(g.work + ((int64_t)blockIdx.y * g.M + m) * ldp + n) = acc[i][j];
      }
    }
    return;
  }
  float scale[MI];
#pragma unroll
  for (int i = 0; i < MI; ++i) scale[i] = row_scale(g, m0 + wm * (BM / 2) + i * 16 + lrow);
  with_scales(scale, [&](auto large) {
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int n = n0 + wn * (BN / 2) + j * 16 + 4 * lgrp;
      const Columns c = columns_at(g, n);
#pragma unroll
      for (int i = 0; i < MI; ++i) store4(g, m0 + wm * (BM / 2) + i * 16 + lrow, n, finished<large>(g, acc[i][j], scale[i], c));
    }
  });
#endif
}

// Few rows: bound by reading B once.  A workgroup takes 16 rows of B, its wavefronts take turns along the contraction, STEP k-tiles at a time whose loads are
// all under way together, from memory straight into the fragments' registers; the parts are added up at the end.  MF fragments of 16 rows of A.
// 1 x 4096 x 4096 5.4 us, 2.5 of them the launch.
template <int MF, int STEP>
__global__ __launch_bounds__(1024) void integer_rows_kernel(const IntegerProductArgs g) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, waves = blockDim.x >> 6, lgrp = lane >> 4, lrow = lane & 15;
  const int n0 = blockIdx.x * 16, nk = (g.K + 127) / 128, Kr = (g.K + 15) & ~15;
  const int ra = g.M < 16 * MF ? g.M : 16 * MF, rb = g.N - n0 < 16 ? g.N - n0 : 16;
  const __amdgpu_buffer_rsrc_t rsrcA = rsrc_of(g.a, (ra - 1) * g.lda + Kr), rsrcB = rsrc_of(g.b + n0 * g.ldb, (rb - 1) * g.ldb + Kr);
  uint32_t oa[MF];                               // rows past the end read as zeros
#pragma unroll
  for (int i = 0; i < MF; ++i) oa[i] = 16 * i + lrow < ra ? (uint32_t)((16 * i + lrow) * g.lda + lgrp * 16) : kOutOfRange;
  const uint32_t ob = lrow < rb ? (uint32_t)(lrow * g.ldb + lgrp * 16) : kOutOfRange;
  i32x4 acc[MF];
#pragma unroll
  for (int i = 0; i < MF; ++i) acc[i] = i32x4{0, 0, 0, 0};
  auto sixteen = [&](__amdgpu_buffer_rsrc_t r, uint32_t row, int k) {       // bytes k + 16 lgrp .. of a row, zeros past K
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, k + lgrp * 16 < Kr && row != kOutOfRange ? row + (uint32_t)k : kOutOfRange, 0, 0));
  };
  for (int k0 = w * STEP; k0 < nk; k0 += waves * STEP) {
    u32x4 b[STEP][2], a[STEP][MF][2];
#pragma unroll
    for (int s = 0; s < STEP; ++s)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = (k0 + s) * 128 + h * 64;
        b[s][h] = sixteen(rsrcB, ob, k);
#pragma unroll
        for (int i = 0; i < MF; ++i) a[s][i][h] = sixteen(rsrcA, oa[i], k);
      }
    if ((g.K & 15) && k0 + STEP >= nk) {
#pragma unroll
      for (int s = 0; s < STEP; ++s)
#pragma unroll
        for (int h = 0; h < 2; ++h) b[s][h] &= first_bytes(g.K - (k0 + s) * 128 - h * 64 - lgrp * 16);
    }
#pragma unroll
    for (int s = 0; s < STEP; ++s)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < MF; ++i) acc[i] = mfma(b[s][h], a[s][i][h], acc[i]);
  }
  i32x4* const part = (i32x4*)smem;
#pragma unroll
  for (int i = 0; i < MF; ++i) part[(i * waves + w) * 64 + lane] = acc[i];
  __syncthreads();
  for (int i = w; i < MF; i += waves) {
    i32x4 sum = part[i * waves * 64 + lane];
    for (int v = 1; v < waves; ++v) sum += part[(i * waves + v) * 64 + lane];
    store4(g, 16 * i + lrow, n0 + 4 * lgrp, finished<true>(g, sum, row_scale(g, 16 * i + lrow), columns_at(g, n0 + 4 * lgrp)));
  }
#endif
}

// Large products (long_tile.h).  Bound by the matrix unit: 8192 x 16384 x 16384 with scales, bias and ReLU 1.51 to 1.6 ms, 2.75 to 2.9 POP/s; the vendor's plain integers 2.1 to 2.2.
template <bool RAGGED>
__global__ __launch_bounds__(256) void integer_long_kernel(const IntegerProductArgs g) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  int tm, tn;
  big_tile(g.M, g.N, tm, tn);
  const int m0 = tm * 256, n0 = tn * 256;
  i32x4 acc[8][8];
  long_tile<i32x4, RAGGED>(acc, smem, g.a + (int64_t)m0 * g.lda, g.b + (int64_t)n0 * g.ldb, g.lda, g.ldb, g.M - m0 < 256 ? g.M - m0 : 256, g.N - n0 < 256 ? g.N - n0 : 256, g.K);
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, wm = w & 1, wn = w >> 1, lgrp = lane >> 4, lrow = lane & 15;
  const int rowW = m0 + wm * 128, colW = n0 + wn * 128;

  // A wavefront stages its 128 x 128 outputs in a 32 KB of the stages that is its own, float32 64 rows at a time, in rows of 256 or 512 bytes whose
  // 16-byte piece c sits at c ^ (row mod 16), and writes whole row segments.
  float scale[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) scale[i] = row_scale(g, rowW + i * 16 + lrow);
  __syncthreads();
  unsigned char* const st = smem + w * 32768;
  with_scales(scale, [&](auto large) {
    if (g.out_dtype == 0) {
      const int c = lane & 31, n = colW + 4 * c;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const Columns col = columns_at(g, colW + j * 16 + 4 * lgrp);
#pragma unroll
          for (int i = 4 * half; i < 4 * half + 4; ++i) {
            asm volatile("" : "+a"(acc[i][j]));
            *(f32x4*)(st + ((i & 3) * 16 + lrow) * 512 + (((4 * j + lgrp) ^ lrow) << 4)) = finished<large>(g, acc[i][j], scale[i], col);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
#pragma unroll
        for (int b0 = 0; b0 < 32; b0 += 8) {
          f32x4 val[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const int r = (b0 + q) * 2 + (lane >> 5);
            val[q] = *(const f32x4*)(st + r * 512 + ((c ^ (r & 15)) << 4));
          }
#pragma unroll
          for (int q = 0; q < 8; ++q) store4(g, rowW + 64 * half + (b0 + q) * 2 + (lane >> 5), n, val[q]);
        }
      }
      return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const Columns col = columns_at(g, colW + j * 16 + 4 * lgrp);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        asm volatile("" : "+a"(acc[i][j]));
        const f32x4 v = finished<large>(g, acc[i][j], scale[i], col);
        const bf16x4 o = {(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
        *(u32x2*)(st + (i * 16 + lrow) * 256 + (((2 * j + (lgrp >> 1)) ^ lrow) << 4) + (lgrp & 1) * 8) = __builtin_bit_cast(u32x2, o);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    const int c = lane & 15, n = colW + 8 * c;
    if (n < g.N) {
      bf16* const out = (bf16*)g.out + (int64_t)rowW * g.ldo + n;
#pragma unroll
      for (int b0 = 0; b0 < 32; b0 += 8) {
        bf16x8 val[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int r = (b0 + q) * 4 + lgrp;
          val[q] = *(const bf16x8*)(st + r * 256 + ((c ^ (r & 15)) << 4));
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int r = (b0 + q) * 4 + lgrp;
          if (rowW + r < g.M) {
            if (n + 8 <= g.N) ((AnyBf16x8*)(out + r * g.ldo))->v = val[q];
            else
              for (int e = 0; e < g.N - n; ++e) out[r * g.ldo + e] = val[q][e];
          }
        }
      }
    }
  });
#endif
}

// The parts of a split contraction added up, then scales, bias, ReLU and rounding.
__global__ __launch_bounds__(256) void integer_join_kernel(const IntegerProductArgs g, int parts) {
  const int quads = (g.N + 3) / 4;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int m = (int)(at / quads), n = (int)(at % quads) * 4;
  if (at >= (int64_t)g.M * quads) return;
  const int64_t ldp = (int64_t)quads * 4;
  i32x4 sum = {0, 0, 0, 0};
  for (int p = 0; p < parts; ++p) sum += *(const i32x4*)(g.work + ((int64_t)p * g.M + m) * ldp + n);
  store4(g, m, n, finished<true>(g, sum, row_scale(g, m), columns_at(g, n)));
}

// ---- host side -------------------------------------------------------------------------------
template <int BM, int BN, int NS, int NG>
hipError_t launch_tile(const IntegerProductArgs& g, int wanted, hipStream_t s) {
  constexpr int smem = NG * NS * (BM + BN) * 128;
  static_assert(smem >= (NG - 1) * BM * BN * 4, "room for the groups' sums");
  static std::atomic<uint64_t> done{0};
  hipError_t e = allow_lds((const void*)integer_tile_kernel<BM, BN, NS, NG>, smem, done);
  if (e != hipSuccess) return e;
  const int nk = (g.K + 127) / 128, all = wanted * NG, kper = all > 1 ? (nk + all - 1) / all : nk, parts = wanted > 1 ? (nk + NG * kper - 1) / (NG * kper) : 1;
  hipLaunchKernelGGL((integer_tile_kernel<BM, BN, NS, NG>), dim3((unsigned)tiles_of(g.M, g.N, BM, BN), parts), dim3(256 * NG), smem, s, g, kper);
  e = hipGetLastError();
  if (e != hipSuccess || parts == 1) return e;
  const int64_t quads = (int64_t)g.M * ((g.N + 3) / 4);
  integer_join_kernel<<<(unsigned)((quads + 255) / 256), 256, 0, s>>>(g, parts);
  return hipGetLastError();
}

template <bool RAGGED>
hipError_t launch_long(const IntegerProductArgs& g, hipStream_t s) {
  static std::atomic<uint64_t> done{0};
  const hipError_t e = allow_lds((const void*)integer_long_kernel<RAGGED>, kLongSmem, done);
  if (e != hipSuccess) return e;
  integer_long_kernel<RAGGED><<<(unsigned)tiles_of(g.M, g.N, 256, 256), 256, kLongSmem, s>>>(g);
  return hipGetLastError();
}

template <int MF, int STEP>
hipError_t launch_rows(const IntegerProductArgs& g, hipStream_t s) {
  const int steps = ((g.K + 127) / 128 + STEP - 1) / STEP, waves = steps > 16 ? 16 : steps > 1 ? steps : 1;
  integer_rows_kernel<MF, STEP><<<(unsigned)((g.N + 15) / 16), waves * 64, MF * waves * 1024, s>>>(g);
  return hipGetLastError();
}

template <typename T, int LANES, int NV, bool LONG>
hipError_t launch_team(const IntegersArgs& a, hipStream_t s) {
  constexpr int teams = 256 / LANES;
  quantize_integers_kernel<T, LANES, NV, LONG><<<(unsigned)(((int64_t)a.rows + teams - 1) / teams), 256, 0, s>>>(a);
  return hipGetLastError();
}
// The smallest team that holds a row.
template <typename T>
hipError_t launch_rows_of(const IntegersArgs& a, hipStream_t s) {
  if (a.cols <= 128) return launch_team<T, 16, 1, false>(a, s);
  if (a.cols <= 512) return launch_team<T, 64, 1, false>(a, s);
  if (a.cols <= 1024) return launch_team<T, 64, 2, false>(a, s);
  if (a.cols <= 2048) return launch_team<T, 256, 1, false>(a, s);
  if (a.cols <= 4096) return launch_team<T, 256, 2, false>(a, s);
  if (a.cols <= 8192) return launch_team<T, 256, 4, false>(a, s);
  if (a.cols <= 16384) return launch_team<T, 256, 8, false>(a, s);
  return launch_team<T, 256, 1, true>(a, s);
}

// The choice of the 8-bit floating-point forms, whose k-tiles take the same time; but few rows whose contraction would be split over workgroups stay whole, on more
// stages: 8 x 16384 x 16384 54.6 (split) / 45.9 us, 20 x 16384 x 8192 28.6 / 25.1.
Shape integer_shape(int M, int N, int K) {
  const Shape s = shape_of(M, N, K, 1, true);
  return s == kSplit && M <= 32 && tiles_of(M, N, 32, 32) > 256 ? k32 : s;
}

}  // namespace

hipError_t launch_quantize_integers(int dtype, const IntegersArgs& a, hipStream_t s) {
  return dtype == 1 ? launch_rows_of<bf16>(a, s) : launch_rows_of<float>(a, s);
}

size_t integer_product_words(int M, int N, int K) {
  const Shape shape = integer_shape(M, N, K);
  if (shape != kSplit && shape != kSplit32by4) return 0;
  const int parts = parts_of(shape, M, N, K);
  return parts > 1 ? (size_t)parts * M * ((N + 3) & ~3) : 0;
}

hipError_t launch_integer_product(const IntegerProductArgs& g, hipStream_t s) {
  const Shape shape = integer_shape(g.M, g.N, g.K);
  const int nk = (g.K + 127) / 128;
  switch (shape) {
    case kRows:
      return g.M <= 16 ? launch_rows<1, 2>(g, s) : launch_rows<2, 2>(g, s);
    case kBig: return g.K & 15 ? launch_long<true>(g, s) : launch_long<false>(g, s);
    case k128: return launch_tile<128, 128, 2, 1>(g, 1, s);
    case k128x64: return launch_tile<128, 64, 2, 1>(g, 1, s);
    case k64: return launch_tile<64, 64, 2, 1>(g, 1, s);
    // One workgroup for each compute unit at most: a third stage is free and hides more of a load.  256 x 4096 x 4096 13.8 / 10.9 us, 48 x 16384 x 4096 19.8 / 16.3; 32x32 48 x
    // 4096 x 8192 15.6 / 10.9, 64 x 4096 x 4096 8.7 / 7.2, 200 x 800 x 3001 6.6 / 6.1.
    case k64by2: return tiles_of(g.M, g.N, 64, 64) <= 256 ? launch_tile<64, 64, 3, 2>(g, 1, s) : launch_tile<64, 64, 2, 2>(g, 1, s);
    case k32x64: return launch_tile<32, 64, 3, 1>(g, 1, s);
    case k32x64by2: return launch_tile<32, 64, 3, 2>(g, 1, s);
    case k32: return nk >= 64 ? launch_tile<32, 32, 6, 1>(g, 1, s) : launch_tile<32, 32, 4, 1>(g, 1, s);
    case k32by4: return nk >= 16 ? launch_tile<32, 32, 3, 4>(g, 1, s) : launch_tile<32, 32, 2, 4>(g, 1, s);
    case kSplit: return launch_tile<64, 64, 3, 1>(g, parts_of(shape, g.M, g.N, g.K), s);
    default: return launch_tile<32, 32, 2, 4>(g, parts_of(shape, g.M, g.N, g.K), s);
  }
}

}  // namespace slp
