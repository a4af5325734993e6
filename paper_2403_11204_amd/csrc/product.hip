// Products of 8-bit matrices with a scale for each block of 128 along the contraction:
//
//   out[m][n] = act(sum over blocks kb of 2^(sa[m][kb] - 127) 2^(sb[n][kb] - 127) sum over k in kb of a[m][k] b[n][k] + bias[n])
//
// Both operands are contraction-contiguous, as in the float32 and bf16 products: forward A W^T, data gradient dZ (W^T)^T, weight gradient
// dZ^T (A^T)^T, the transposed copies made where the values are quantised.
//
// Two forms of the multiplication:
//   * bf16 outputs: v_mfma_scale_f32_16x16x128_f8f6f4 multiplies a 16 x 16 block over 128 k, exactly a scale's block, multiplies by both scales
//     and adds in float32: the scales cost no vector instruction and the sums never leave the accumulators (that is why the scales are
//     powers of two).  Inside the instruction, as inside every 8-bit one of this chip, the products of 8 consecutive k are lined up with the largest of
//     them and cut off 13 bits below the power of two that its factors' exponents make; the sums of 8 are then added with 24 bits.  A product of 7
//     beside one of 65536 is lost, and at most 7 times 2^-13 of the largest product of each 8 is.  On normal values that is 1.4e-5 of the result's norm, 6e-5 on
//     values spread over e^1.5, whatever the length, where rounding the output to bf16 costs 1.7e-3.  A register-only loop of it runs at 3700-4400 TFLOP/s.
//   * float32 outputs (gradients of weights above all), bf16 ones whose caller asks for float32 sums, and products of few rows: the values are turned
//     into bf16, scale and all, which is exact between 2^-126 and 1.75 2^127 (4 of 8 bits are used; scales from 2^-117 to 2^119 keep every value there.  Above, a value
//     becomes infinite, which 256 2^120 is in float32 as well; below, it loses bits and ends as zero under 2^-133), and
//     v_mfma_f32_16x16x32_bf16 adds the exact products in float32: 1.7e-8 and 7e-8 on the same values, at 2100-2200 TFLOP/s.
//
// A lane feeds either form 32 bytes of one row, as two 16-byte pieces of the row's 128: both operands take the same two pieces, so which k an
// instruction pairs with which lane does not matter.  The operands are passed in the order B, A: a lane then holds 4 consecutive
// columns of one row of the output.
#include "eightbit_device.h"

#include <atomic>
#include <type_traits>
#include <utility>

namespace slp {
namespace {

constexpr int kXcds = 8;
constexpr uint32_t kOutOfRange = 0x80000000u;     // byte offset past the end of every tile
#define SLP_VMCNT(n) ((((n) & 15) | 0x0F70 | (((n) >> 4) << 14)))
#define SLP_VMCNT_LGKM0(n) (SLP_VMCNT(n) & 0xF0FF)

// A lane's 32 values of a fragment and the scale of its row, as either form takes them.
template <bool EXACT> struct Fragment;
template <> struct Fragment<false> {
  i32x8 v;
  int scale;
  __device__ __forceinline__ void set(const i32x8& bytes, int s) {
    v = bytes;
    scale = s;
  }
};
template <> struct Fragment<true> {
  bf16x8 v[4];
  __device__ __forceinline__ void set(const i32x8& bytes, int s) {
    const float scale = scale_value((uint32_t)s);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)bytes[i], scale, false);
      const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)bytes[i], scale, true);
      v[i >> 1][4 * (i & 1)] = lo[0];
      v[i >> 1][4 * (i & 1) + 1] = lo[1];
      v[i >> 1][4 * (i & 1) + 2] = hi[0];
      v[i >> 1][4 * (i & 1) + 3] = hi[1];
    }
  }
};
__device__ __forceinline__ f32x4 mma(const Fragment<false>& b, const Fragment<false>& a, const f32x4& acc) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b.v, a.v, acc, 0, 0, 0, b.scale, 0, a.scale);
}
__device__ __forceinline__ f32x4 mma(const Fragment<true>& b, const Fragment<true>& a, f32x4 acc) {
#pragma unroll
  for (int q = 0; q < 4; ++q) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.v[q], a.v[q], acc, 0, 0, 0);
  return acc;
}

// What lies between a row's last column and the next multiple of 16 is whatever the memory holds (the columns that follow, where the matrix is part of a
// wider one).  It is read with the last piece of the row, and cut off with this: ones over the first n of 16 bytes.
__device__ __forceinline__ u32x4 first_bytes(int n) {
  u32x4 mask;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = n - 4 * i;
    mask[i] = m >= 4 ? ~0u : m <= 0 ? 0u : (1u << (8 * m)) - 1u;
  }
  return mask;
}
// The same for a lane's two pieces of a k-tile of which `left` columns exist; what begins past them is zero already.
__device__ __forceinline__ void cut_off(i32x8& v, int left, int lgrp) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int n = left - 64 * h - 16 * lgrp;
    const u32x4 mask = first_bytes(n);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[4 * h + j] &= (int)mask[j];
  }
}

// Four consecutive columns n .. n + 3 of row m.
__device__ __forceinline__ void store4(const ProductArgs& g, int m, int n, f32x4 v) {
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
__device__ __forceinline__ f32x4 finished(const ProductArgs& g, f32x4 v, f32x4 bias) {
  const float least = g.relu ? 0.0f : -INFINITY;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = __builtin_elementwise_maximum(v[e] + bias[e], least);       // (a NaN stays one)
  return v;
}
// bias[n .. n + 3]; what is past its end is the last one, for columns that nobody stores
__device__ __forceinline__ f32x4 bias4(const ProductArgs& g, int n) {
  f32x4 b = {0.0f, 0.0f, 0.0f, 0.0f};
  if (g.bias) {
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = g.bias[n + e < g.N ? n + e : g.N - 1];
  }
  return b;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_of(const void* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00020000);
}

// BM x BN tile, 4 wavefronts in a 2 x 2 grid, NS LDS stages of a k-tile of 128 each, one barrier a k-tile.  NG such groups of wavefronts
// take a part of the contraction each (kper k-tiles) and are added up in order at the end.  blockIdx.y: part of the contraction of a whole workgroup;
// several parts leave float32 partial products for join_kernel.  1000 x 3001 x 1500, 752 tiles of 64x64: bf16 11.7 us, float32 17.2 (520 TFLOP/s; contractions of 1504 16.1): operands
// into LDS 5.6 us of it, conversions and matrix instructions 4.5 each, 2.5 the launch.  1024 x 4096 x 4096 on 128x64: bf16 24.8 (1.39 PFLOP/s), float32 40.3.
template <int BM, int BN, int NS, int NG, bool EXACT>
__global__ __launch_bounds__(256 * NG) void product_tile_kernel(const ProductArgs g, int kper) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ __attribute__((aligned(16))) unsigned char all_smem[];
  constexpr int A_BYTES = BM * 128, STAGE = (BM + BN) * 128, SCALES = NS * STAGE;        // behind the stages a ring of two groups of scales
  const int group = NG > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) : 0;
  unsigned char* const smem = all_smem + group * (SCALES + 2048);
  constexpr int LA = BM / 32, LB = BN / 32, NLD = LA + LB;                               // loads a lane per k-tile
  constexpr int MI = BM / 32, NI = BN / 32;
  constexpr int AW = (BM + 63) / 64, BW = (BN + 63) / 64;                                // wavefronts that load A's and B's scales
  static_assert(AW + BW <= 4, "one load of scales per wavefront");
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
  // scales: for every 4 k-tiles wavefront w loads the dwords that hold theirs for 64 of the tile's rows, A's and then B's, ahead of the first's
  // data.  A load at every k-tile takes 2 to 5 % longer (1000 x 3001 x 1500 in float32 16.8 us / 16.2 here)
  const bool sA = w < AW;
  const int srow = 64 * (sA ? w : w - AW) + lane;
  const int sm = sA ? m0 : n0, sshift = sA ? g.shift_a : g.shift_b, sfirst = sm >> sshift;
  const int64_t slds = sA ? g.ldsa : g.ldsb;
  const int slast = ((sm + (sA ? ra : rb) - 1) >> sshift) - sfirst;
  const __amdgpu_buffer_rsrc_t rsrcS = rsrc_of((sA ? g.sa : g.sb) + sfirst * slds, slast * slds + ((nk + 3) & ~3));
  const uint32_t soff = srow < (sA ? ra : rb) ? (uint32_t)((((sm + srow) >> sshift) - sfirst) * slds) : kOutOfRange;

  typedef __attribute__((address_space(3))) void* lds_ptr_t;
  const int lds_wave = __builtin_amdgcn_readfirstlane(w * 1024), lds_scale = __builtin_amdgcn_readfirstlane(SCALES + w * 256);
  auto load = [&](int kt, int stage) {
    unsigned char* const st = smem + stage * STAGE;
    const bool in = kt < k1, in_k = in && kt * 128 + chunk * 16 < Kr;
    const uint32_t koff = (uint32_t)kt * 128u;
    if ((kt & 3) == 0)                 // (k0 is a multiple of 4, too)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrcS, (lds_ptr_t)(smem + lds_scale + (kt & 4) * 256), 4, in && soff != kOutOfRange ? soff + (uint32_t)kt : kOutOfRange, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < LA + LB; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(i < LA ? rsrcA : rsrcB, (lds_ptr_t)(st + lds_wave + i * 4096), 16,
                                               in_k && voff[i] != kOutOfRange ? voff[i] + koff : kOutOfRange, 0, 0, 0);
  };
  const uint32_t fragA = (uint32_t)((wm * (BM / 2) + lrow) * 128), fragB = (uint32_t)(A_BYTES + (wn * (BN / 2) + lrow) * 128);
  const uint32_t x0 = (uint32_t)((lgrp ^ ((lane >> 1) & 7)) << 4), x1 = x0 ^ 64;
  const uint32_t scaleA = (uint32_t)(SCALES + (wm * (BM / 2) + lrow) * 4), scaleB = (uint32_t)(SCALES + AW * 256 + (wn * (BN / 2) + lrow) * 4);

  f32x4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  // a k-tile that everybody's loads have filled
  auto multiply = [&](int kt, auto ragged) {
    const unsigned char* const st = smem + (kt - k0) % NS * STAGE;
    const unsigned char* const sc = smem + (kt & 4) * 256 + (kt & 3);
    Fragment<EXACT> a[MI], b[NI];
    auto fragment = [&](uint32_t at) {
      const u32x4 lo = *(const u32x4*)(st + at + x0), hi = *(const u32x4*)(st + at + x1);
      i32x8 v = {(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
      if constexpr (ragged) cut_off(v, g.K & 127, lgrp);
      return v;
    };
#pragma unroll
    for (int j = 0; j < NI; ++j) b[j].set(fragment(fragB + j * 2048), sc[scaleB + j * 64]);
#pragma unroll
    for (int i = 0; i < MI; ++i) a[i].set(fragment(fragA + i * 2048), sc[scaleA + i * 64]);
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = mma(b[j], a[i], acc[i][j]);
  };
#pragma unroll
  for (int s = 0; s < NS - 1; ++s) load(k0 + s, s);
  // The last k-tile has a copy of its own behind the loop where it ends inside 16 bytes: 0.2 to 0.3 us of such a product (1000 x 3001 x 1500 in float32 16.9 / 17.2, its
  // sums then leave nothing to the memory behind a row's end).  Asked inside the loop, every product would take 0.2 us longer.
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
    f32x4* const sums = (f32x4*)all_smem + t;
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

#pragma unroll
  for (int j = 0; j < NI; ++j) {
    const int n = n0 + wn * (BN / 2) + j * 16 + 4 * lgrp;
    if (gridDim.y > 1) {
      const int64_t ldp = (g.N + 3) & ~3;
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const int m = m0 + wm * (BM / 2) + i * 16 + lrow;
        if (m < g.M && n < g.N) *(f32x4*)(g.work + ((int64_t)blockIdx.y * g.M + m) * ldp + n) = acc[i][j];
      }
    } else {
      const f32x4 bias = bias4(g, n);
#pragma unroll
      for (int i = 0; i < MI; ++i) store4(g, m0 + wm * (BM / 2) + i * 16 + lrow, n, finished(g, acc[i][j], bias));
    }
  }
#endif
}

// Few rows (a request's, a short last batch): bound by reading B once.  A workgroup takes 16 rows of B, its wavefronts take turns along the
// contraction, STEP k-tiles at a time whose loads are all under way together, from memory straight into the fragments' registers; the parts are
// added up in the order of the wavefronts.  MF fragments of 16 rows of A.  Both output types take the exact form: the conversions hide behind
// the loads.  Microseconds on the device, this kernel / tiles: 1 x 4096 x 4096 5.2 / 6.5 (16.8 MB from caches at 6 TB/s behind 2.5 us of launch and
// latency), 4 x 16384 x 16384 50.3 / 55.6 (5.4 TB/s), 8 x 4096 x 4096 6.1 / 6.5.  32 rows of B a workgroup, which halves the reading of A: 1 x 4096 x
// 4096 7.0, 1 x 16384 x 16384 52.1 (47.5 with 16).
template <int MF, int STEP>
__global__ __launch_bounds__(1024) void product_rows_kernel(const ProductArgs g) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, waves = blockDim.x >> 6, lgrp = lane >> 4, lrow = lane & 15;
  const int n0 = blockIdx.x * 16, nk = (g.K + 127) / 128, Kr = (g.K + 15) & ~15;
  const int ra = g.M < 16 * MF ? g.M : 16 * MF, rb = g.N - n0 < 16 ? g.N - n0 : 16;
  const int sfirst = n0 >> g.shift_b, sblocks = ((n0 + rb - 1) >> g.shift_b) - sfirst;
  const __amdgpu_buffer_rsrc_t rsrcA = rsrc_of(g.a, (ra - 1) * g.lda + Kr), rsrcB = rsrc_of(g.b + n0 * g.ldb, (rb - 1) * g.ldb + Kr);
  const __amdgpu_buffer_rsrc_t rsrcSA = rsrc_of(g.sa, ((ra - 1) >> g.shift_a) * g.ldsa + nk), rsrcSB = rsrc_of(g.sb + sfirst * g.ldsb, sblocks * g.ldsb + nk);
  // rows past the end read as zeros, under a scale of zero
  uint32_t oa[MF], osa[MF];
#pragma unroll
  for (int i = 0; i < MF; ++i) {
    const int m = 16 * i + lrow;
    oa[i] = m < ra ? (uint32_t)(m * g.lda + lgrp * 16) : kOutOfRange;
    osa[i] = m < ra ? (uint32_t)((m >> g.shift_a) * g.ldsa) : kOutOfRange;
  }
  const uint32_t ob = lrow < rb ? (uint32_t)(lrow * g.ldb + lgrp * 16) : kOutOfRange;
  const uint32_t osb = lrow < rb ? (uint32_t)((((n0 + lrow) >> g.shift_b) - sfirst) * g.ldsb) : kOutOfRange;
  f32x4 acc[MF];
#pragma unroll
  for (int i = 0; i < MF; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  auto sixteen = [&](__amdgpu_buffer_rsrc_t r, uint32_t row, int k) {       // bytes k + 16 lgrp .. of a row, zeros past K
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, k + lgrp * 16 < Kr ? row + (uint32_t)k : kOutOfRange, 0, 0));
  };
  auto piece = [&](__amdgpu_buffer_rsrc_t r, uint32_t row, int kt) {
    const u32x4 lo = sixteen(r, row, kt * 128), hi = sixteen(r, row, kt * 128 + 64);
    return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };
  auto scale = [&](__amdgpu_buffer_rsrc_t r, uint32_t row, int kt) {        // (past the end: the last one, for zeros)
    return (int)(uint8_t)__builtin_amdgcn_raw_buffer_load_b8(r, row + (uint32_t)(kt < nk ? kt : nk - 1), 0, 0);
  };
  auto turn = [&](int k0, auto ragged) {
    i32x8 vb[STEP], va[STEP][MF];
    int sb[STEP], sa[STEP][MF];
#pragma unroll
    for (int s = 0; s < STEP; ++s) {
      vb[s] = piece(rsrcB, ob, k0 + s);
      sb[s] = scale(rsrcSB, osb, k0 + s);
#pragma unroll
      for (int i = 0; i < MF; ++i) {
        va[s][i] = piece(rsrcA, oa[i], k0 + s);
        sa[s][i] = scale(rsrcSA, osa[i], k0 + s);
      }
    }
#pragma unroll
    for (int s = 0; s < STEP; ++s) {
      Fragment<true> b, a;
      if constexpr (ragged) cut_off(vb[s], g.K - (k0 + s) * 128, lgrp);
      b.set(vb[s], sb[s]);
#pragma unroll
      for (int i = 0; i < MF; ++i) {
        if constexpr (ragged) cut_off(va[s][i], g.K - (k0 + s) * 128, lgrp);
        a.set(va[s][i], sa[s][i]);
        acc[i] = mma(b, a, acc[i]);
      }
    }
  };
  // a copy of its own for the turn that ends inside 16 bytes: the question alone takes 0.2 us of every call
  int k0 = w * STEP;
  for (const int end = g.K & 15 ? nk - STEP : nk; k0 < end; k0 += waves * STEP) turn(k0, std::false_type{});
  if (k0 < nk) turn(k0, std::true_type{});
  f32x4* const part = (f32x4*)smem;
#pragma unroll
  for (int i = 0; i < MF; ++i) part[(i * waves + w) * 64 + lane] = acc[i];
  __syncthreads();
  for (int i = w; i < MF; i += waves) {
    f32x4 sum = part[i * waves * 64 + lane];
    for (int v = 1; v < waves; ++v) sum += part[(i * waves + v) * 64 + lane];
    store4(g, 16 * i + lrow, n0 + 4 * lgrp, finished(g, sum, bias4(g, n0 + 4 * lgrp)));
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
__device__ __forceinline__ void big_tile(const ProductArgs& g, int& tm, int& tn) {
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

// Large products: a 256x256 tile on 4 wavefronts of 128 x 128, one on each SIMD, accumulators in 256 AGPRs, two LDS stages of 64 KB, a k-tile
// of 128 (one scale).  8192 x 16384 x 16384: bf16 1460-1500 us (2.9-3.0 PFLOP/s; 2576 cycles a k-tile, 2048 of them MFMAs, at the clock that the power limit
// leaves), float32 2860-2940 (1.5 PFLOP/s, 5355 cycles of 4096), 8192 x 8192 x 4096 float32 387 us.  One wavefront on a SIMD has nobody to fill its issue slots, so everything else goes between the MFMAs, a few
// instructions at a time.  The scales of 4 k-tiles come as one dword for each row into a ring of two, and from there as a byte beside
// each fragment.  MFMAs and loads are assembly: the accumulators stay where they are, and a load's LDS address (m0) is set in front of an MFMA.
//
// bf16 outputs: a k-tile is 64 MFMAs of 32 cycles, in 4 strips of 2 A fragments against all 8 B fragments.  B's fragments stay in
// registers for the whole k-tile; A's are read a strip ahead.
//   strip 1  barrier X: nobody reads this k-tile's B rows any more;  strips 1, 2: the 8 loads of k-tile kt + 2 into them
//   strip 3  barrier Y: k-tile kt + 1 has landed, nobody reads this one's A rows;  strips 3, 0: the 8 loads of kt + 2 into those;
//            strips 3 and 0 read kt + 1's B fragments, one every third MFMA, each behind the last that uses its predecessor and 6 ahead of
//            the first that uses it
// The loop starts at strip 1, where the compiler, which waits for every LDS read at a loop's head, finds only those that strip needs.
//
// float32 outputs (EXACT): a k-tile is 2 sub-steps of 64 k, each 128 bf16 MFMAs of 16 cycles in the same 4 strips.  Both operands pass through a
// conversion on the way, 128 of them a sub-step, one behind each MFMA: B's fragments, double-buffered, behind the even ones, A's, a strip
// ahead, behind the odd ones; the bytes are read from LDS 14 MFMAs before their conversion starts.
//   sub-step 1, MFMA   0  barrier Z: k-tile kt + 1 has landed, nobody reads this one's B rows;  4 .. 60: the 8 loads of kt + 2 into them
//                     72  barrier X: nobody reads this one's A rows;  76 .. 132 (into the next sub-step): the 8 loads of kt + 2 into those
constexpr int kBigScales = 2 * 512 * 128, kBigSmem = kBigScales + 2 * 512 * 4;
template <bool EXACT>
__global__ __launch_bounds__(256) void product_long_kernel(const ProductArgs g) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef __attribute__((ext_vector_type(4))) int i32x4;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int A_BYTES = 256 * 128, STAGE = 512 * 128;
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
  // scales: wavefront w loads rows 64 w .. 64 w + 63 of A's and of B's
  const int srow = 64 * w + lane, sfA = m0 >> g.shift_a, sfB = n0 >> g.shift_b, slA = ((m0 + ra - 1) >> g.shift_a) - sfA, slB = ((n0 + rb - 1) >> g.shift_b) - sfB;
  const i32x4 rsrcSA = rsrc(g.sa + sfA * g.ldsa, slA * g.ldsa + ((nk + 3) & ~3)), rsrcSB = rsrc(g.sb + sfB * g.ldsb, slB * g.ldsb + ((nk + 3) & ~3));
  const uint32_t soffA = srow < ra ? (uint32_t)((((m0 + srow) >> g.shift_a) - sfA) * g.ldsa) : kOutOfRange;
  const uint32_t soffB = srow < rb ? (uint32_t)((((n0 + srow) >> g.shift_b) - sfB) * g.ldsb) : kOutOfRange;
  typedef __attribute__((address_space(3))) void* lds_ptr_t;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)smem;
  const uint32_t lds_wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(lds0 + w * 1024));
  const uint32_t lds_scale = (uint32_t)__builtin_amdgcn_readfirstlane((int)(lds0 + kBigScales + w * 256));

  f32x4 acc[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

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
#define SLP_LOAD_ARGS(i, base_, koff_)                                                                                             \
  [base] "s"(base_), [row] "i"((i) < 8 ? (i) * 4096 : A_BYTES + ((i) - 8) * 4096), [off] "v"(voff[i]), [rsrc] "s"((i) < 8 ? rsrcA : rsrcB), \
      [koff] "s"(koff_)
  auto load = [&](int i, uint32_t base, uint32_t koff) {
    asm volatile("s_add_u32 m0, %[base], %[row]\n\ts_nop 1\n\tbuffer_load_dwordx4 %[off], %[rsrc], %[koff] offen lds"
                 : : SLP_LOAD_ARGS(i, base, koff) : "memory", "scc", "m0");
  };
  auto load_scales = [&](int group) {
    const uint32_t at = lds_scale + (group & 1) * 2048, koff = (uint32_t)(group * 4 < nk ? group * 4 : 0);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 1\n\tbuffer_load_dword %1, %2, %3 offen lds" : : "s"(at), "v"(soffA), "s"(rsrcSA), "s"(koff) : "memory", "m0");
    asm volatile("s_add_u32 m0, %0, 0x400\n\ts_nop 1\n\tbuffer_load_dword %1, %2, %3 offen lds" : : "s"(at), "v"(soffB), "s"(rsrcSB), "s"(koff) : "memory", "scc", "m0");
  };
  const uint32_t x0 = (uint32_t)((lgrp ^ ((lane >> 1) & 7)) << 4), x1 = x0 ^ 64;       // a lane's two pieces of a row
  const uint32_t fa = (uint32_t)((wm * 128 + lrow) * 128), fb = (uint32_t)(A_BYTES + (wn * 128 + lrow) * 128);
  const uint32_t fsa = (uint32_t)(kBigScales + (wm * 128 + lrow) * 4), fsb = (uint32_t)(kBigScales + (256 + wn * 128 + lrow) * 4);
  auto scale_at = [&](int kt) {                  // k-tile nk takes the last one's: zeros times any scale of the row's own
    const int k = kt < nk ? kt : nk - 1;
    return (uint32_t)((k >> 2 & 1) * 2048 + (k & 3));
  };
  // pair m of a sub-step's fragments: strip m / 16; columns forwards, but backwards in strip 1, so that mostly one operand changes from one
  // to the next
  constexpr auto col_of = [](int m) { return m / 16 == 1 ? 7 - m % 16 / 2 : m % 16 / 2; };
  constexpr auto row_of = [](int m) { return 2 * (m / 16) + ((m / 2 & 1) ? 1 - m % 2 : m % 2); };
#define SLP_FENCE() __builtin_amdgcn_sched_barrier(0)
#define SLP_BARRIER(cnt)                                            \
  do {                                                              \
    asm volatile("" ::: "memory");                                  \
    __builtin_amdgcn_s_waitcnt(cnt);                                \
    asm volatile("" ::: "memory");                                  \
    __builtin_amdgcn_s_barrier();                                   \
    asm volatile("" ::: "memory");                                  \
  } while (0)
  // The k-tile whose last piece ends inside 16 bytes: a lane cuts off what it has loaded itself, `wait` having seen it land, before the barrier behind which
  // others read it.  Only the last k-tiles' copy of the loop asks: the question in the loop itself takes 1 %.
  const int ragged = g.K & 15 ? nk - 1 : -1;
#define SLP_CUT(kt, wait)                                                                                           \
  do {                                                                                                              \
    if ((kt) == ragged) {                                                                                           \
      __builtin_amdgcn_s_waitcnt(wait);                                                                             \
      asm volatile("" ::: "memory");                                                                                \
      if (chunk == (g.K >> 4 & 7)) {                                                                                \
        const u32x4 mask = first_bytes(g.K & 15);                                                                   \
        u32x4* const p = (u32x4*)(smem + ((kt) & 1) * STAGE + w * 1024 + lane * 16);                                \
        _Pragma("unroll 4") for (int i = 0; i < 16; ++i) p[i * 256] &= mask;                                        \
      }                                                                                                             \
      asm volatile("" ::: "memory");                                                                                \
      __builtin_amdgcn_s_waitcnt(0xC07F);                                                                           \
    }                                                                                                               \
  } while (0)
  const int whole = ragged < 0 ? nk : nk < 2 ? 0 : nk - 2;       // k-tiles in front of the last two
  const int rowW = m0 + wm * 128, colW = n0 + wn * 128;
  f32x4 bias[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) bias[j] = bias4(g, colW + j * 16 + 4 * lgrp);
  // k-tiles 0 and 1 and the first group of scales; the last 4 loads of A's rows of k-tile 1 go out beside the first MFMAs
  clip(0);
  load_scales(0);
  static_for<16>([&](auto i) { load(i, lds_wave, 0u); });
  clip(1);
  static_for<8>([&](auto i) { load(8 + i, lds_wave + STAGE, koff_of(1)); });

  if constexpr (!EXACT) {
  static_for<4>([&](auto i) { load(i, lds_wave + STAGE, koff_of(1)); });
  i32x8 a[4], b[8];              // A fragments of strips with even and odd number, 2 each
  int sa[4], sb[8];
  auto bytes = [&](int stage, uint32_t at) {
    const u32x4 lo = *(const u32x4*)(smem + stage * STAGE + at + x0), hi = *(const u32x4*)(smem + stage * STAGE + at + x1);
    return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };
  auto read_a = [&](int kt, int f) {             // fragment f of the 8
    const int r = f & 3;
    a[r] = bytes(kt & 1, fa + f * 2048);
    sa[r] = smem[fsa + scale_at(kt) + f * 64];
  };
  auto read_b = [&](int kt, int f) {
    b[f] = bytes(kt & 1, fb + f * 2048);
    sb[f] = smem[fsb + scale_at(kt) + f * 64];
  };
#define SLP_MFMA "v_mfma_scale_f32_16x16x128_f8f6f4 %[acc], %[b], %[a], %[acc], %[sb], %[sa] op_sel_hi:[0,0,0]"
#define SLP_MFMA_ARGS(i, j) [b] "v"(b[j]), [a] "v"(a[(i) & 3]), [sb] "v"(sb[j]), [sa] "v"(sa[(i) & 3])
  auto mma = [&](int i, int j) { asm volatile(SLP_MFMA : [acc] "+a"(acc[i][j]) : SLP_MFMA_ARGS(i, j)); };
  // where the compiler may have touched a scale just before: an MFMA reads what a vector instruction wrote two instructions later at the earliest
  auto mma_first = [&](int i, int j) { asm volatile("s_nop 1\n\t" SLP_MFMA : [acc] "+a"(acc[i][j]) : SLP_MFMA_ARGS(i, j)); };
  auto mma_load = [&](int i, int j, int l, uint32_t base, uint32_t koff) {        // the MFMA is the wait state that m0 needs
    asm volatile("s_add_u32 m0, %[base], %[row]\n\t" SLP_MFMA "\n\tbuffer_load_dwordx4 %[off], %[rsrc], %[koff] offen lds"
                 : [acc] "+a"(acc[i][j]) : SLP_MFMA_ARGS(i, j), SLP_LOAD_ARGS(l, base, koff) : "memory", "scc", "m0");
  };
  // strip S of k-tile kt; loads go to k-tile kl
  auto strip = [&](auto sc, int kt, int kl) {
    constexpr int S = decltype(sc)::value;
    const uint32_t base = lds_wave + (kl & 1) * STAGE, koff = koff_of(kl);
    static_for<16>([&](auto pc) {
      constexpr int p = decltype(pc)::value, m = 16 * S + p, i = row_of(m), j = col_of(m);
      // fragments: A's of the next strip, B's and the first of A's of the next k-tile in strip 3
      if constexpr (S < 3 && (p == 2 || p == 5)) read_a(kt, 2 * S + 2 + (p == 5));
      if constexpr (S == 3 && (p == 1 || p == 3)) read_a(kt + 1, p == 3);
      if constexpr (S == 3 && p % 3 == 2) read_b(kt + 1, p / 3);
      if constexpr (S == 0 && p % 3 == 1 && p < 8) read_b(kt, 5 + p / 3);
      constexpr int l = (S == 1 || S == 2) ? 8 + (S - 1) * 4 + p / 4 : (S == 3 ? 0 : 4) + p / 4;
      if constexpr (p % 4 == 2) mma_load(i, j, l, base, koff);
      else if constexpr (p < 2) mma_first(i, j);
      else mma(i, j);
      SLP_FENCE();
    });
  };
  constexpr std::integral_constant<int, 0> s0{};
  constexpr std::integral_constant<int, 1> s1{};
  constexpr std::integral_constant<int, 2> s2{};
  constexpr std::integral_constant<int, 3> s3{};

  SLP_CUT(0, SLP_VMCNT(12));
  SLP_BARRIER(SLP_VMCNT(12));
#pragma unroll
  for (int f = 0; f < 5; ++f) read_b(0, f);
  read_a(0, 0);
  read_a(0, 1);
  strip(s0, 0, 1);
  auto ktile = [&](int kt, auto last) {
    SLP_BARRIER(0xC07F);                                   // X: every LDS read so far has returned
    clip(kt + 2);
    if ((kt & 3) == 0) load_scales(kt / 4 + 1);
    SLP_FENCE();
    strip(s1, kt, kt + 2);
    strip(s2, kt, kt + 2);
    if constexpr (last) SLP_CUT(kt + 1, SLP_VMCNT(8));
    SLP_BARRIER(SLP_VMCNT_LGKM0(8));                       // Y
    strip(s3, kt, kt + 2);
    strip(s0, kt + 1, kt + 2);                             // (of k-tile nk, too: all zeros)
  };
  int kt = 0;
  for (; kt < whole; ++kt) ktile(kt, std::false_type{});
  for (; kt < nk; ++kt) ktile(kt, std::true_type{});
#undef SLP_MFMA
#undef SLP_MFMA_ARGS
  } else {
  bf16x8 a[2][2][2], b[2][8][2];           // [strip's or sub-step's parity][fragment][32 k]
  u32x4 rawa[2], rawb[2];
  int sa[2], sb[2];
  // bytes of fragment f of sub-step kk of k-tile kt
  auto read_a = [&](int kt, int kk, int f) {
    rawa[f & 1] = *(const u32x4*)(smem + (kt & 1) * STAGE + fa + f * 2048 + (kk ? x1 : x0));
    sa[f & 1] = smem[fsa + scale_at(kt) + f * 64];
  };
  auto read_b = [&](int kt, int kk, int f) {
    rawb[f & 1] = *(const u32x4*)(smem + (kt & 1) * STAGE + fb + f * 2048 + (kk ? x1 : x0));
    sb[f & 1] = smem[fsb + scale_at(kt) + f * 64];
  };
  // conversion e of the 8 of a fragment: 2 values, with their scale (the instruction reads its exponent's bits)
  auto convert = [&](const u32x4& raw, int scale, bf16x8 (&to)[2], auto ec) {
    constexpr int e = decltype(ec)::value;
    const bf16x2 v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(raw[e / 2], scale_value((uint32_t)scale), e % 2 == 1);
    to[e / 4][2 * (e % 4)] = v[0];
    to[e / 4][2 * (e % 4) + 1] = v[1];
  };
#define SLP_MFMA "v_mfma_f32_16x16x32_bf16 %[acc], %[b], %[a], %[acc]"
#define SLP_MFMA_ARGS(kk, i, j, q) [b] "v"(b[kk][j][q]), [a] "v"(a[(i) / 2 & 1][(i) & 1][q])
  auto mma = [&](int kk, int i, int j, int q) { asm volatile(SLP_MFMA : [acc] "+a"(acc[i][j]) : SLP_MFMA_ARGS(kk, i, j, q)); };
  auto mma_load = [&](int kk, int i, int j, int q, int l, uint32_t base, uint32_t koff) {
    asm volatile("s_add_u32 m0, %[base], %[row]\n\t" SLP_MFMA "\n\tbuffer_load_dwordx4 %[off], %[rsrc], %[koff] offen lds"
                 : [acc] "+a"(acc[i][j]) : SLP_MFMA_ARGS(kk, i, j, q), SLP_LOAD_ARGS(l, base, koff) : "memory", "scc", "m0");
  };
  // Sub-step KK of k-tile kt.  MFMA p: pair p / 2, 32 k p % 2.
  auto substep = [&](auto kc, int kt, auto last) {
    constexpr int KK = decltype(kc)::value;
    const int kn = KK ? kt + 1 : kt;               // k-tile of the next sub-step
    const uint32_t base0 = lds_wave + ((kt & 1) ^ 1) * STAGE, koff0 = koff_of(kt + 1), base1 = lds_wave + (kt & 1) * STAGE, koff1 = koff_of(kt + 2);
    static_for<128>([&](auto pc) {
      constexpr int p = decltype(pc)::value, i = row_of(p / 2), j = col_of(p / 2), q = p % 2, S = p / 32;
      if constexpr (KK == 1 && p == 0) {
        if constexpr (last) SLP_CUT(kt + 1, SLP_VMCNT(0));
        SLP_BARRIER(SLP_VMCNT_LGKM0(0));                                           // Z
      }
      if constexpr (KK == 1 && p == 2) clip(kt + 2);
      if constexpr (KK == 1 && p == 72) SLP_BARRIER(0xC07F);                       // X
      // bytes: B's of the next sub-step, A's of the strip after the next (14 MFMAs ahead of the conversions)
      if constexpr (p % 16 == 0) read_b(kn, KK ^ 1, p / 16);
      if constexpr (p % 16 == 3 || p % 32 == 19) {
        constexpr int f = 2 * S + (p % 32 == 19 ? 4 : 3);                          // fragments 3 .. 10: 8, 9 and 10 are the next sub-step's 0, 1 and 2
        if constexpr (f < 8) read_a(kt, KK, f);
        else read_a(kn, KK ^ 1, f - 8);
      }
      constexpr bool loads = KK == 1 ? (p >= 4 && p <= 60 && p % 8 == 4) || (p >= 76 && p % 8 == 4) : p == 4;
      if constexpr (!loads) mma(KK, i, j, q);
      else if constexpr (KK == 0) mma_load(KK, i, j, q, 7, base0, koff0);
      else if constexpr (p <= 60) mma_load(KK, i, j, q, 8 + (p - 4) / 8, base1, koff1);
      else mma_load(KK, i, j, q, (p - 76) / 8, base1, koff1);
      if constexpr (p % 2 == 0) {
        constexpr int at = p - 14 >= 0 ? p - 14 : p - 14 + 128, f = at / 16, e = at % 16 / 2;
        if constexpr (p >= 14) convert(rawb[f & 1], sb[f & 1], b[KK ^ 1][f], std::integral_constant<int, e>{});
        else convert(rawb[f & 1], sb[f & 1], b[KK][f], std::integral_constant<int, e>{});        // the current sub-step's last fragment
      } else {
        constexpr int f = p % 32 / 16, e = p % 16 / 2;
        convert(rawa[f], sa[f], a[(S + 1) & 1][f], std::integral_constant<int, e>{});
      }
      SLP_FENCE();
    });
  };
  constexpr std::integral_constant<int, 0> k0{};
  constexpr std::integral_constant<int, 1> k1{};
  static_for<7>([&](auto i) { load(i, lds_wave + STAGE, koff_of(1)); });
  SLP_CUT(0, SLP_VMCNT(15));
  SLP_BARRIER(SLP_VMCNT(15));
  // what a sub-step finds: B's fragments but the last one's conversions, the first strip of A's, the bytes of the fragment behind each
  static_for<7>([&](auto f) {
    read_b(0, 0, f);
    static_for<8>([&](auto e) { convert(rawb[f & 1], sb[f & 1], b[0][f], e); });
  });
  read_b(0, 0, 7);
  static_for<1>([&](auto) { convert(rawb[1], sb[1], b[0][7], std::integral_constant<int, 0>{}); });
  static_for<2>([&](auto f) {
    read_a(0, 0, f);
    static_for<8>([&](auto e) { convert(rawa[f], sa[f], a[0][f], e); });
  });
  read_a(0, 0, 2);
  SLP_FENCE();
  auto ktile = [&](int kt, auto last) {
    if ((kt & 3) == 0) load_scales(kt / 4 + 1);
    SLP_FENCE();
    substep(k0, kt, last);
    substep(k1, kt, last);
  };
  int kt = 0;
  for (; kt < whole; ++kt) ktile(kt, std::false_type{});
  for (; kt < nk; ++kt) ktile(kt, std::true_type{});
  }
  // the last zero fills have landed, and the matrix pipe is done with the accumulators (the compiler does not see MFMAs in assembly)
  __builtin_amdgcn_s_waitcnt(SLP_VMCNT_LGKM0(0));
  asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
  for (int i = 0; i < 64; ++i) asm volatile("" : "+a"(acc[i / 8][i % 8]));
#undef SLP_FENCE
#undef SLP_BARRIER
#undef SLP_CUT
#undef SLP_LOAD_ARGS
#undef SLP_MFMA
#undef SLP_MFMA_ARGS
#pragma clang diagnostic pop

  // A wavefront stages its 128 x 128 outputs in a 32 KB of the stages that is its own, float32 64 rows at a time, in rows of 256 or 512 bytes whose
  // 16-byte piece c sits at c ^ (row mod 16), and writes whole row segments.
  __syncthreads();
  unsigned char* const st = smem + w * 32768;
  if constexpr (EXACT) {
    const int c = lane & 31, n = colW + 4 * c;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
#pragma unroll
        for (int i = 4 * half; i < 4 * half + 4; ++i) {
          asm volatile("" : "+a"(acc[i][j]));
          *(f32x4*)(st + ((i & 3) * 16 + lrow) * 512 + (((4 * j + lgrp) ^ lrow) << 4)) = finished(g, acc[i][j], bias[j]);
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
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      asm volatile("" : "+a"(acc[i][j]));
      const f32x4 v = finished(g, acc[i][j], bias[j]);
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

// The parts of a split contraction added up in order, then bias, ReLU and rounding.
__global__ __launch_bounds__(256) void join_kernel(const ProductArgs g, int parts) {
  const int quads = (g.N + 3) / 4;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int m = (int)(at / quads), n = (int)(at % quads) * 4;
  if (at >= (int64_t)g.M * quads) return;
  const int64_t ldp = (int64_t)quads * 4;
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int p = 0; p < parts; ++p) sum += *(const f32x4*)(g.work + ((int64_t)p * g.M + m) * ldp + n);
  store4(g, m, n, finished(g, sum, bias4(g, n)));
}

// ---- host side -------------------------------------------------------------------------------
int64_t tiles_of(int M, int N, int BM, int BN) { return (int64_t)((M + BM - 1) / BM) * ((N + BN - 1) / BN); }

// Which kernel a product runs on.
enum Shape { kRows, kBig, k128, k128x64, k64, k64by2, k32x64, k32x64by2, k32, k32by4, kSplit, kSplit32by4 };

// Whether it is product_rows_kernel.  Its workgroups read A as often as there are 16 rows of B, and a compute unit reads 16 rows in 0.7 us per
// 1024 k (1.2 with 16 rows of A).  Microseconds, this / tiles: 1 x 1000 x 784 2.9 / 3.9, 1 x 4096 x 8192 8.2 / 10.9, 4 x 512 x 8192 8.0 / 7.7, 1 x 1000 x
// 16384 12.3 / 8.7, 12 x 4096 x 4096 6.6 / 6.5, 8 x 2048 x 8192 9.6 / 8.1, 16 x 1000 x 2000 4.5 / 4.9, 16 x 1000 x 4000 6.9 / 6.4, 32 x 4096 x 1024 4.1 / 4.3,
// 32 x 1000 x 2000 5.7 / 5.0; with 4 fragments of A 40 x 1000 x 784 4.5 / 4.1, 64 x 64 x 256 3.6 / 3.0, 64 x 1000 x 784 4.8 / 4.1;
// many columns 16 x 16384 x 1024 6.4 / 5.5, 32 x 16384 x 512 5.6 / 4.7.
bool few_rows(int M, int N, int K) {
  if (M <= 4) return K <= 8192 || N >= 4096;
  return M <= 32 && (int64_t)M * K <= 32768 && (N + 63) / 64 < 192;
}

// All microseconds on the device, operands in the caches.  256x256 tiles where they keep most of the 256 compute units busy, sooner with a bf16
// output, whose k-tiles are half as long: 1700 x 6000 x 2000 (168 tiles) 28.7 against 37.5 on smaller ones, 3000 x 3000 x 1000 (144) 20.4 / 20.1, 2048 x
// 4096 x 4096 (128) 45 / 39; float32 3000 x 3000 x 1000 33.6 / 28.8, 2472 x 4096 x 2700 (160) 65.3 / 65.3;
// short contractions with a float32 output, which are all stores: 4096 x 8192 x 64 42 / 33, 256 45 / 40, 512 57 / 54, 784 68 / 75;
// the same with a bf16 output whose rows are not on 16 bytes, 256 at most: 581 x 14917 x 256 24.8 / 14.0, 581 x 14914 x 256 17.7 / 12.4, on 16 bytes 2048 x 8192 x 256 15.7 /
// 18.4, 8192 x 8192 x 256 51 / 62;
// and not where most of a tile would lie past a side (60000 rows, 1024 k): 10 columns 26.6 / 12.1, float32 38.6 / 13.9, 100 columns 30.6 / 17.3, 34.5 / 22.8; 200
// columns 22.8 / 28.8, 35.0 / 40.3.
// Where there is less than one tile for a compute unit, a k-tile's steps (barrier, LDS, conversion, product) wait for one another; two or four groups of
// wavefronts with a part of the contraction each fill the gaps, as long as a part is long enough.  32x32 in one group / four: 300 x 300 x 1000 4.8 / 5.1, x 1400
// 5.7 / 5.4, 200 x 800 x 3001 9.5 / 7.6, 714 x 174 x 4096 10.2 (split, two launches) / 8.3; 32x64 in one / two: 1000 x 512 x 500 4.7 / 5.2, x 800 5.9 / 5.6, x 2048 9.2
// / 7.8, x 4096 15.8 (split) / 12.0; 64x64 in one / two: 1000 x 1000 x 500 5.9 / 6.3, x 800 7.3 / 6.9, x 4096 21.3 (split) / 15.7, bf16 16.8 / 10.8; 1200 x 1200 x 1500
// (361 tiles) 11.9 / 12.5, x 3000 19.8 / 18.2, bf16 15.1 / 12.6.  At 64x64 as long as all workgroups are on the chip together: 7759 x 234 x 8192 (488) bf16 36.0 / 27.7, 1500 x
// 1500 x 4096 (576) 20.6 / 26.9.  A very long contraction is split over workgroups, too: 64 x 64 x 16384 in one / split 22.1 / 12.5, split
// on 32x32 in four groups 9.8; 128 x 512 x 8192 12.8 / 11.5 / 9.3; 300 x 300 x 6200 (100 of these tiles) 11.5 / 12.0 / 10.8, 784 x 128 x 60000 (100) 86 / 31 / 50;
// in one / split 247 x 1024 x 8192 (256) bf16 10.0 / 14.6, 256 x 1024 x 12000 19.8 / 17.2, 200 x 800 x 8192 13.0 / 14.7, 200 x 400 x 12000 12.6 / 11.6; 1000 x 512 x 6200 (512) 17.4 / 19.4,
// x 8192 21.0 / 20.0, 1000 x 1000 x 8192 bf16 24.6 / 21.4.
// Otherwise the smallest tiles that leave each compute unit one workgroup: 32x32 against 32x64 and 64x64 on 226 x 679 x 837 (176 tiles) 4.5 / 5.1 / 5.8, 462 x 1024 x
// 146 (480) 4.0 / 3.8 / 4.2, 618 x 1341 x 256 (840) 5.4 / 4.5 / 4.4.  Larger ones as soon as they fill the chip, of which a compute unit holds 4 (64x64), 3
// (128x64) and 2 (128x128): 64x64 against 128x64 on 491 x 5192 x 24 (328 of the latter) 6.3 / 7.0, 392 x 4096 x 540 (256) 7.8 / 8.5, 436 x 8192 x 2512 (512) 20.1 /
// 16.6; 128x64 against 128x128 on 2048 x 4096 x 1024 (512 of the latter) 18.1 / 15.9, 1024 x 8192 x 8192 (512) 102 / 69, 3000 x 3000 x 1000 float32 (576)
// 28.8 / 32.9, 440 x 10342 x 324 (324) 8.6 / 10.5.
// form: 0 converts to bf16 (float32 outputs and float32 sums), 1 is the scaled instruction.
Shape shape_of(int M, int N, int K, int form, bool aligned) {
  const int nk = (K + 127) / 128;
  if (few_rows(M, N, K)) return kRows;
  if ((M < N ? M : N) > 128 && K > (form == 1 && aligned ? 0 : 256) && tiles_of(M, N, 256, 256) >= (form == 1 ? 144 : 192)) return kBig;
  const int64_t t64 = tiles_of(M, N, 64, 64), t32 = tiles_of(M, N, 32, 32);
  if (nk >= (t32 <= 64 ? 48 : t32 <= 256 ? 80 : 60) && t64 <= 256) return t32 <= 64 ? kSplit32by4 : kSplit;
  if (t32 <= 256) return nk >= 11 ? k32by4 : k32;
  if (tiles_of(M, N, 32, 64) <= 256) return nk >= 7 ? k32x64by2 : k32x64;
  if (nk >= 7 && t64 <= (nk >= 32 ? 512 : nk >= 16 ? 384 : 256)) return k64by2;
  if (tiles_of(M, N, 128, 64) < 480) return k64;
  const int64_t t128 = tiles_of(M, N, 128, 128);
  return t128 >= 384 && t128 <= 512 && nk >= 4 ? k128 : k128x64;
}

// Parts of a split contraction: two workgroups for each compute unit, 8 k-tiles at least (1000 x 512 x 8192, 128 tiles, in 2, 4 and 8 parts 22.7, 20.6, 23.0
// us); one with four groups of wavefronts, 16 k-tiles at least.
int parts_of(Shape shape, int M, int N, int K) {
  const int nk = (K + 127) / 128;
  const int64_t t = shape == kSplit ? 512 / tiles_of(M, N, 64, 64) : 256 / tiles_of(M, N, 32, 32);
  const int most = shape == kSplit ? nk / 8 : nk / 16;
  return t < most ? (int)t : most;
}

// Lets a kernel have that much LDS, once on each device (bit of `done`); host threads that launch first together both do.
hipError_t allow_lds(const void* kernel, int bytes, std::atomic<uint64_t>& done) {
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return e;
  const uint64_t bit = (uint64_t)1 << (device & 63);
  if (device < 64 && (done.load(std::memory_order_acquire) & bit)) return hipSuccess;
  e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess && device < 64) done.fetch_or(bit, std::memory_order_release);
  return e;
}

template <int BM, int BN, int NS, int NG, bool EXACT>
hipError_t launch_tile(const ProductArgs& g, int wanted, hipStream_t s) {
  constexpr int smem = NG * (NS * (BM + BN) * 128 + 2048);
  static_assert(smem >= (NG - 1) * BM * BN * 4, "room for the groups' sums");
  static std::atomic<uint64_t> done{0};
  hipError_t e = allow_lds((const void*)product_tile_kernel<BM, BN, NS, NG, EXACT>, smem, done);
  if (e != hipSuccess) return e;
  const int nk = (g.K + 127) / 128, all = wanted * NG, kper = all > 1 ? ((nk + all - 1) / all + 3) & ~3 : nk, parts = wanted > 1 ? (nk + NG * kper - 1) / (NG * kper) : 1;
  hipLaunchKernelGGL((product_tile_kernel<BM, BN, NS, NG, EXACT>), dim3((unsigned)tiles_of(g.M, g.N, BM, BN), parts), dim3(256 * NG), smem, s, g, kper);
  e = hipGetLastError();
  if (e != hipSuccess || parts == 1) return e;
  const int64_t quads = (int64_t)g.M * ((g.N + 3) / 4);
  join_kernel<<<(unsigned)((quads + 255) / 256), 256, 0, s>>>(g, parts);
  return hipGetLastError();
}

template <bool EXACT>
hipError_t launch_long(const ProductArgs& g, hipStream_t s) {
  static std::atomic<uint64_t> done{0};
  const hipError_t e = allow_lds((const void*)product_long_kernel<EXACT>, kBigSmem, done);
  if (e != hipSuccess) return e;
  product_long_kernel<EXACT><<<(unsigned)tiles_of(g.M, g.N, 256, 256), 256, kBigSmem, s>>>(g);
  return hipGetLastError();
}

template <int MF, int STEP>
hipError_t launch_rows(const ProductArgs& g, hipStream_t s) {
  const int steps = ((g.K + 127) / 128 + STEP - 1) / STEP, waves = steps > 16 ? 16 : steps > 1 ? steps : 1;
  product_rows_kernel<MF, STEP><<<(unsigned)((g.N + 15) / 16), waves * 64, MF * waves * 1024, s>>>(g);
  return hipGetLastError();
}

template <bool EXACT>
hipError_t launch_shape(const ProductArgs& g, Shape shape, hipStream_t s) {
  switch (shape) {
    case kRows:
      return g.M <= 16 ? launch_rows<1, 2>(g, s) : launch_rows<2, 2>(g, s);
    case kBig: return launch_long<EXACT>(g, s);
    case k128: return launch_tile<128, 128, 2, 1, EXACT>(g, 1, s);
    case k128x64: return launch_tile<128, 64, 2, 1, EXACT>(g, 1, s);
    case k64: return launch_tile<64, 64, 2, 1, EXACT>(g, 1, s);
    case k64by2: return launch_tile<64, 64, 2, 2, EXACT>(g, 1, s);
    case k32x64: return launch_tile<32, 64, 3, 1, EXACT>(g, 1, s);
    case k32x64by2: return launch_tile<32, 64, 3, 2, EXACT>(g, 1, s);
    case k32: return launch_tile<32, 32, 4, 1, EXACT>(g, 1, s);
    case k32by4: return launch_tile<32, 32, 2, 4, EXACT>(g, 1, s);
    case kSplit: return launch_tile<64, 64, 3, 1, EXACT>(g, parts_of(shape, g.M, g.N, g.K), s);
    default: return launch_tile<32, 32, 2, 4, EXACT>(g, parts_of(shape, g.M, g.N, g.K), s);
  }
}

}  // namespace

// (of the larger one for the two forms)
size_t product_floats(int M, int N, int K) {
  int parts = 1;
  for (int form = 0; form < 2; ++form) {
    const Shape shape = shape_of(M, N, K, form, true);       // (no product of 144 such tiles is split)
    if (shape != kSplit && shape != kSplit32by4) continue;
    const int p = parts_of(shape, M, N, K);
    parts = p > parts ? p : parts;
  }
  return parts > 1 ? (size_t)parts * M * ((N + 3) & ~3) : 0;
}

hipError_t launch_product(const ProductArgs& g, hipStream_t s) {
  const bool exact = g.exact || g.out_dtype == 0;
  const Shape shape = shape_of(g.M, g.N, g.K, exact ? 0 : 1, (((uintptr_t)g.out / 2 | g.ldo) & 7) == 0);
  return exact ? launch_shape<true>(g, shape, s) : launch_shape<false>(g, shape, s);
}

}  // namespace slp
