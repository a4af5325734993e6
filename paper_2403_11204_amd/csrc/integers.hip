// 8-bit integers with a scale for each row (a token of the activations, an output channel of the weights):
//
//   q = round(127 x / max|x|), scale = max|x| / 127;   out[m][n] = act(sa[m] sb[n] sum over k of a[m][k] b[n][k] + bias[n])
//
// The sums are integers, exact whatever the order: contractions of up to 131071 stay below 2^31.  v_mfma_i32_16x16x64_i8 does 64 k of a 16 x 16 block in 16
// cycles, as much as the 8-bit floating-point forms.  Operands are laid out, loaded and passed (in the order B, A: a lane holds 4 consecutive columns of one
// row of the output) as in product.hip; with nothing to convert and no scales on the way, a k-tile is reads and matrix instructions only.
#include "eightbit_device.h"
#include "gemm_launch.h"
#include "product_shapes.h"

#include <type_traits>
#include <utility>

namespace slp {
namespace {

constexpr int kXcds = 8;
constexpr uint32_t kOutOfRange = 0x80000000u;     // byte offset past the end of every tile
#define SLP_VMCNT(n) ((((n) & 15) | 0x0F70 | (((n) >> 4) << 14)))
#define SLP_VMCNT_LGKM0(n) (SLP_VMCNT(n) & 0xF0FF)
typedef __attribute__((ext_vector_type(4))) int i32x4;

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
// length.  Bound by memory: one reading, one writing of a byte for each element.
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

// What lies between a row's last column and the next multiple of 16 is whatever the memory holds.  It is read with the last piece of the row, and cut off
// one operand with this: ones over the first n of 16 bytes.
__device__ __forceinline__ u32x4 first_bytes(int n) {
  u32x4 mask;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = n - 4 * i;
    mask[i] = m >= 4 ? ~0u : m <= 0 ? 0u : (1u << (8 * m)) - 1u;
  }
  return mask;
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
__device__ __forceinline__ f32x4 finished(const IntegerProductArgs& g, const i32x4& sum, float scale, const Columns& c) {
  const float least = g.relu ? 0.0f : -INFINITY;
  f32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = __builtin_elementwise_maximum((float)sum[e] * scale * c.scale[e] + c.bias[e], least);       // (a NaN stays one)
  return v;
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
// leave partial sums for integer_join_kernel.
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
#pragma unroll
  for (int j = 0; j < NI; ++j) {
    const int n = n0 + wn * (BN / 2) + j * 16 + 4 * lgrp;
    const Columns c = columns_at(g, n);
#pragma unroll
    for (int i = 0; i < MI; ++i) store4(g, m0 + wm * (BM / 2) + i * 16 + lrow, n, finished(g, acc[i][j], scale[i], c));
  }
#endif
}

// Few rows: bound by reading B once.  A workgroup takes 16 rows of B, its wavefronts take turns along the contraction, STEP k-tiles at a time whose loads are
// all under way together, from memory straight into the fragments' registers; the parts are added up at the end.  MF fragments of 16 rows of A.
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
    store4(g, 16 * i + lrow, n0 + 4 * lgrp, finished(g, sum, row_scale(g, 16 * i + lrow), columns_at(g, n0 + 4 * lgrp)));
  }
#endif
}

// f(0), f(1), ... f(N - 1) with the index as a constant.
template <typename F, int... I>
__device__ __forceinline__ void static_for_impl(F f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, typename F>
__device__ __forceinline__ void static_for(F f) { static_for_impl(f, std::make_integer_sequence<int, N>{}); }

// workgroup -> 256x256 tile.  Consecutive workgroups go round the XCDs: all of them work on one 16 x 16 region of tiles at a time where
// the tiles divide into such, on contiguous runs of tile columns 8 tiles high otherwise.
__device__ __forceinline__ void big_tile(const IntegerProductArgs& g, int& tm, int& tn) {
  const int tilesM = (g.M + 255) / 256, tilesN = (g.N + 255) / 256, pid = blockIdx.x, xcd = pid % kXcds, q = pid / kXcds;
  if (tilesM % 16 == 0 && tilesN % 16 == 0) {
    const int r = q / 32, sl = q % 32, regions = tilesM / 16;
    tm = (r % regions) * 16 + (xcd % 2) * 8 + sl % 8;
    tn = (r / regions) * 16 + (xcd / 2) * 4 + sl / 8;
    return;
  }
  const int total = tilesM * tilesN, base = total / kXcds, rem = total % kXcds, tid = xcd * base + (xcd < rem ? xcd : rem) + q;
  const int width = 8 * tilesN, first = tid / width * 8, rows = tilesM - first < 8 ? tilesM - first : 8;
  tm = first + tid % width % rows;
  tn = tid % width / rows;
}

// The order in which a sub-step's 8 A fragments meet its 8 B fragments: strips of two rows, down the columns and back, so that from one matrix instruction to the
// next one operand changes.
struct Walk {
  int a[64], b[64], first[16];     // fragments of instruction m; all fragments (0 .. 7 A, 8 .. 15 B) in the order of their first use
  constexpr Walk() : a(), b(), first() {
    for (int m = 0; m < 64; ++m) {
      const int strip = m / 16, c = m % 16 / 2;
      a[m] = 2 * strip + (c & 1 ? 1 - m % 2 : m % 2);
      b[m] = strip & 1 ? 7 - c : c;
    }
    bool seen[16] = {};
    for (int m = 0, n = 0; m < 64; ++m)
      for (int f : {a[m], 8 + b[m]})
        if (!seen[f]) {
          seen[f] = true;
          first[n++] = f;
        }
  }
};

// Large products: a 256x256 tile on 4 wavefronts of 128 x 128, one on each SIMD, accumulators in 256 AGPRs, two LDS stages of 64 KB, a k-tile of 128 bytes.  A
// k-tile is 128 matrix instructions of 16 cycles, two sub-steps of 64 k whose 16 fragments are in registers before they start; everything else goes between
// them, at most two instructions at a time:
//   instruction   0 ..  30   reads of sub-step 1
//                40          barrier X: nobody reads this k-tile's stage any more
//                42 .. 132   the 16 loads of k-tile kt + 2 into that stage (the last one in the next k-tile's time)
//                79          barrier Y: k-tile kt + 1 has landed
//                80 .. 125   reads of its sub-step 0
// Matrix instructions and loads are assembly: the accumulators stay where they are, and a load's LDS address (m0) is set in front of a matrix instruction.
// RAGGED: the contraction ends inside 16 bytes.
constexpr int kBigSmem = 2 * 512 * 128;
template <bool RAGGED>
__global__ __launch_bounds__(256) void integer_long_kernel(const IntegerProductArgs g) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int A_BYTES = 256 * 128, STAGE = 512 * 128;
  constexpr int RD1 = 0, X = 40, LD = 42, LD_STEP = 6, Y = 79, RD0 = 80;      // instruction index of what the comment above lists
  constexpr int kOwn = (128 - LD + LD_STEP - 1) / LD_STEP;                    // loads of a k-tile that do not go out in the next one's time
  constexpr int kBeforeY = (Y - LD + LD_STEP - 1) / LD_STEP;                  // loads of k-tile kt + 2 that are out at barrier Y
  static_assert(kOwn <= 16 && LD > X && LD + 15 * LD_STEP - 128 < X && RD1 + 2 * 15 < X && RD0 + 3 * 15 < 128, "order of the events of a k-tile");
  int tm, tn;
  big_tile(g, tm, tn);
  const int m0 = tm * 256, n0 = tn * 256;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, wm = w & 1, wn = w >> 1, lgrp = lane >> 4, lrow = lane & 15;
  const int nk = (g.K + 127) / 128, Kr = (g.K + 15) & ~15;
  const int ra = g.M - m0 < 256 ? g.M - m0 : 256, rb = g.N - n0 < 256 ? g.N - n0 : 256;
  // a buffer resource by words: as an operand of assembly it has to be a vector
  auto rsrc = [](const void* p, int64_t bytes) {
    const uint64_t a = (uint64_t)(uintptr_t)p;
    return i32x4{(int)(uint32_t)a, (int)(uint32_t)(a >> 32), (int)bytes, 0x00020000};
  };
  const i32x4 rsrcA = rsrc(g.a + (int64_t)m0 * g.lda, (ra - 1) * g.lda + Kr), rsrcB = rsrc(g.b + (int64_t)n0 * g.ldb, (rb - 1) * g.ldb + Kr);
  // load i < 8 fills rows [32 i, 32 i + 32) of A's tile, i >= 8 of B's; wavefront w rows 8w .. 8w + 7 of those
  const int prow = w * 8 + (lane >> 3), chunk = (lane & 7) ^ ((prow >> 1) & 7);
  uint32_t voff[16];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    voff[i] = prow + 32 * i < ra ? (uint32_t)((prow + 32 * i) * g.lda + chunk * 16) : kOutOfRange;
    voff[8 + i] = prow + 32 * i < rb ? (uint32_t)((prow + 32 * i) * g.ldb + chunk * 16) : kOutOfRange;
  }
  typedef __attribute__((address_space(3))) void* lds_ptr_t;
  const uint32_t lds_wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(uintptr_t)(lds_ptr_t)smem + w * 1024));
  const int rowW = m0 + wm * 128, colW = n0 + wn * 128;

  i32x4 acc[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = i32x4{0, 0, 0, 0};

  // Chunks past K become zero fills: one that is past it in a k-tile is past it in all that follow.
  auto clip = [&](int kt) {
    if (kt * 128 + 128 > Kr) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (kt * 128 + chunk * 16 >= Kr) voff[i] = kOutOfRange;
    }
  };
  // The k offset is a scalar; k-tiles past the end, whose offsets are out of range already, take 0, so that no sum of the two wraps.
  auto koff_of = [&](int kt) { return (uint32_t)(kt < nk ? kt : 0) * 128u; };
  // The statements name the m0 they set, so that one set by the compiler for an access of its own does not pass for still set behind them; it
  // warns of every register it reserves.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
#define SLP_LOAD "s_add_u32 m0, %[base], %[row]\n\t"
#define SLP_LOAD_ARGS(i, base_, koff_)                                                                                             \
  [base] "s"(base_), [row] "i"((i) < 8 ? (i) * 4096 : A_BYTES + ((i) - 8) * 4096), [off] "v"(voff[i]), [rsrc] "s"((i) < 8 ? rsrcA : rsrcB), \
      [koff] "s"(koff_)
  auto load = [&](int i, uint32_t base, uint32_t koff) {
    asm volatile(SLP_LOAD "s_nop 1\n\tbuffer_load_dwordx4 %[off], %[rsrc], %[koff] offen lds" : : SLP_LOAD_ARGS(i, base, koff) : "memory", "scc", "m0");
  };
  u32x4 af[2][8], bfr[2][8];
  uint32_t fa[2], fb[2];
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    const uint32_t xo = (uint32_t)(((kk * 4 + lgrp) ^ ((lane >> 1) & 7)) << 4);
    fa[kk] = (uint32_t)((wm * 128 + lrow) * 128) + xo;
    fb[kk] = (uint32_t)(A_BYTES + (wn * 128 + lrow) * 128) + xo;
  }
  constexpr Walk walk;
  auto read = [&](int stage, int kk, int f) {
    if (f < 8) af[kk][f] = *(const u32x4*)(smem + stage * STAGE + fa[kk] + f * 2048);
    else bfr[kk][f - 8] = *(const u32x4*)(smem + stage * STAGE + fb[kk] + (f - 8) * 2048);
  };
  auto mma = [&](int kk, int ia, int ib) {
    asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(acc[ia][ib]) : "v"(bfr[kk][ib]), "v"(af[kk][ia]));
  };
  auto mma_load = [&](int kk, int ia, int ib, int i, uint32_t base, uint32_t koff) {        // the matrix instruction is the wait state that m0 needs
    asm volatile(SLP_LOAD "v_mfma_i32_16x16x64_i8 %[acc], %[b], %[a], %[acc]\n\tbuffer_load_dwordx4 %[off], %[rsrc], %[koff] offen lds"
                 : [acc] "+a"(acc[ia][ib]) : [b] "v"(bfr[kk][ib]), [a] "v"(af[kk][ia]), SLP_LOAD_ARGS(i, base, koff) : "memory", "scc", "m0");
  };
#define SLP_FENCE() __builtin_amdgcn_sched_barrier(0)
#define SLP_BARRIER(cnt)                                            \
  do {                                                              \
    asm volatile("" ::: "memory");                                  \
    __builtin_amdgcn_s_waitcnt(cnt);                                \
    asm volatile("" ::: "memory");                                  \
    __builtin_amdgcn_s_barrier();                                   \
    asm volatile("" ::: "memory");                                  \
  } while (0)
  constexpr int kLgkm0 = 0xC07F;         // every LDS read has returned
  // The k-tile whose last piece ends inside 16 bytes: a lane cuts off what it has loaded itself of B's rows, `wait` having seen it land, before the barrier behind
  // which others read it.
  auto cut = [&](int kt, auto wait) {
    if (RAGGED && kt == nk - 1) {
      __builtin_amdgcn_s_waitcnt(decltype(wait)::value);
      asm volatile("" ::: "memory");
      if (chunk == (g.K >> 4 & 7)) {
        const u32x4 mask = first_bytes(g.K & 15);
        u32x4* const p = (u32x4*)(smem + (kt & 1) * STAGE + A_BYTES + w * 1024 + lane * 16);
#pragma unroll 4
        for (int i = 0; i < 8; ++i) p[i * 256] &= mask;
      }
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(kLgkm0);
    }
  };
  clip(0);
  static_for<16>([&](auto i) { load(i, lds_wave, 0u); });
  clip(1);
  static_for<kOwn>([&](auto i) { load(i, lds_wave + STAGE, koff_of(1)); });
  cut(0, std::integral_constant<int, SLP_VMCNT(kOwn)>{});
  SLP_BARRIER(SLP_VMCNT(kOwn));
#pragma unroll
  for (int f = 0; f < 16; ++f) read(0, 0, f);
  for (int kt = 0; kt < nk; ++kt) {
    const int cur = kt & 1, nxt = cur ^ 1;
    const uint32_t base1 = lds_wave + nxt * STAGE, base2 = lds_wave + cur * STAGE, koff1 = koff_of(kt + 1), koff2 = koff_of(kt + 2);
    static_for<128>([&](auto pc) {
      constexpr int p = decltype(pc)::value, kk = p / 64, ia = walk.a[p % 64], ib = walk.b[p % 64], late = p + 128 - LD, own = p - LD;
      if constexpr (p == X) {
        SLP_BARRIER(kLgkm0);
        clip(kt + 2);
      }
      if constexpr (p == Y) {
        cut(kt + 1, std::integral_constant<int, SLP_VMCNT(kBeforeY)>{});
        SLP_BARRIER(SLP_VMCNT(kBeforeY));
      }
      if constexpr (p >= RD1 && (p - RD1) % 2 == 0 && (p - RD1) / 2 < 16) read(cur, 1, walk.first[(p - RD1) / 2]);
      if constexpr (p >= RD0 && (p - RD0) % 3 == 0 && (p - RD0) / 3 < 16) read(nxt, 0, walk.first[(p - RD0) / 3]);
      if constexpr (late % LD_STEP == 0 && late / LD_STEP < 16) mma_load(kk, ia, ib, late / LD_STEP, base1, koff1);
      else if constexpr (own >= 0 && own % LD_STEP == 0 && own / LD_STEP < 16) mma_load(kk, ia, ib, own / LD_STEP, base2, koff2);
      else mma(kk, ia, ib);
      SLP_FENCE();
    });
  }
  // the last zero fills have landed, and the matrix pipe is done with the accumulators (the compiler does not see instructions in assembly)
  __builtin_amdgcn_s_waitcnt(SLP_VMCNT_LGKM0(0));
  asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
  for (int i = 0; i < 64; ++i) asm volatile("" : "+a"(acc[i / 8][i % 8]));
#undef SLP_FENCE
#undef SLP_BARRIER
#undef SLP_LOAD
#undef SLP_LOAD_ARGS
#pragma clang diagnostic pop

  // A wavefront stages its 128 x 128 outputs in a 32 KB of the stages that is its own, float32 64 rows at a time, in rows of 256 or 512 bytes whose
  // 16-byte piece c sits at c ^ (row mod 16), and writes whole row segments.
  float scale[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) scale[i] = row_scale(g, rowW + i * 16 + lrow);
  __syncthreads();
  unsigned char* const st = smem + w * 32768;
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
          *(f32x4*)(st + ((i & 3) * 16 + lrow) * 512 + (((4 * j + lgrp) ^ lrow) << 4)) = finished(g, acc[i][j], scale[i], col);
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
      const f32x4 v = finished(g, acc[i][j], scale[i], col);
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
  store4(g, m, n, finished(g, sum, row_scale(g, m), columns_at(g, n)));
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
  const hipError_t e = allow_lds((const void*)integer_long_kernel<RAGGED>, kBigSmem, done);
  if (e != hipSuccess) return e;
  integer_long_kernel<RAGGED><<<(unsigned)tiles_of(g.M, g.N, 256, 256), 256, kBigSmem, s>>>(g);
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

Shape integer_shape(int M, int N, int K) { return shape_of(M, N, K, 1, true); }

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
  switch (shape) {
    case kRows:
      return g.M <= 16 ? launch_rows<1, 2>(g, s) : launch_rows<2, 2>(g, s);
    case kBig: return g.K & 15 ? launch_long<true>(g, s) : launch_long<false>(g, s);
    case k128: return launch_tile<128, 128, 2, 1>(g, 1, s);
    case k128x64: return launch_tile<128, 64, 2, 1>(g, 1, s);
    case k64: return launch_tile<64, 64, 2, 1>(g, 1, s);
    case k64by2: return launch_tile<64, 64, 2, 2>(g, 1, s);
    case k32x64: return launch_tile<32, 64, 3, 1>(g, 1, s);
    case k32x64by2: return launch_tile<32, 64, 3, 2>(g, 1, s);
    case k32: return launch_tile<32, 32, 4, 1>(g, 1, s);
    case k32by4: return launch_tile<32, 32, 2, 4>(g, 1, s);
    case kSplit: return launch_tile<64, 64, 3, 1>(g, parts_of(shape, g.M, g.N, g.K), s);
    default: return launch_tile<32, 32, 2, 4>(g, parts_of(shape, g.M, g.N, g.K), s);
  }
}

}  // namespace slp
