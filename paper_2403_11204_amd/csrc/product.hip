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
//     powers of two).  Inside the instruction, as inside every 8-bit one of this chip, the products of neighbouring k are lined up with the largest of
//     them and keep about 15 bits below it: measured 1.4e-5 of the result's norm on normal values, 6e-5 on values spread over e^1.5, whatever the
//     length, where rounding the output to bf16 costs 1.7e-3.  A register-only loop of it runs at 3700-4400 TFLOP/s.
//   * float32 outputs (gradients of weights above all): the values are turned into bf16, scale and all, which is exact (4 of 8 bits are used), and
//     v_mfma_f32_16x16x32_bf16 adds the exact products in float32: 1.7e-8 and 7e-8 on the same values, at 2100-2200 TFLOP/s.
//
// A lane feeds either form 32 bytes of one row, as two 16-byte pieces of the row's 128: both operands take the same two pieces, so which k an
// instruction pairs with which lane does not matter.  The operands are passed in the order B, A: a lane then holds 4 consecutive
// columns of one row of the output.
#include "eightbit_device.h"

#include <mutex>

namespace slp {
namespace {

constexpr int kXcds = 8;
constexpr uint32_t kOutOfRange = 0x80000000u;     // byte offset past the end of every tile
#define SLP_VMCNT(n) ((((n) & 15) | 0x0F70 | (((n) >> 4) << 14)))
#define SLP_VMCNT_LGKM0(n) (SLP_VMCNT(n) & 0xF0FF)

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

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
    const float scale = __builtin_bit_cast(float, s << 23);       // the conversion reads the exponent's bits
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
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] += bias[e];
    if (g.relu) v[e] = v[e] < 0.0f ? 0.0f : v[e];       // (a NaN stays one)
  }
  return v;
}
__device__ __forceinline__ f32x4 bias4(const ProductArgs& g, int n) {
  f32x4 b = {0.0f, 0.0f, 0.0f, 0.0f};
  if (g.bias) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < g.N) b[e] = g.bias[n + e];
  }
  return b;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_of(const void* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00020000);
}

// BM x BN tile, 4 wavefronts in a 2 x 2 grid, NS LDS stages of a k-tile of 128 each, one barrier a k-tile.  blockIdx.y: part of the
// contraction (kper k-tiles each); several parts leave float32 partial products for join_kernel.
template <int BM, int BN, int NS, bool EXACT>
__global__ __launch_bounds__(256) void product_tile_kernel(const ProductArgs g, int kper) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int A_BYTES = BM * 128, DATA = (BM + BN) * 128, STAGE = DATA + 4 * 256;      // + a dword of scales for each row
  constexpr int LA = BM / 32, LB = BN / 32, NLD = LA + LB + 1;                           // loads a lane per k-tile
  constexpr int MI = BM / 32, NI = BN / 32;
  static_assert(BM + BN <= 256, "one load of scales per wavefront");
  const int tilesM = (g.M + BM - 1) / BM, tilesN = (g.N + BN - 1) / BN, total = tilesM * tilesN;
  int tid;
  {
    const int pid = blockIdx.x, xcd = pid % kXcds, q = pid / kXcds, base = total / kXcds, rem = total % kXcds;
    tid = xcd * base + (xcd < rem ? xcd : rem) + q;
  }
  constexpr int kGroup = 8;
  const int width = kGroup * tilesN, first = tid / width * kGroup, rows = tilesM - first < kGroup ? tilesM - first : kGroup;
  const int m0 = (first + tid % width % rows) * BM, n0 = tid % width / rows * BN;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, wm = w & 1, wn = w >> 1, lgrp = lane >> 4, lrow = lane & 15;

  const int nk = (g.K + 127) / 128, Kr = (g.K + 15) & ~15;
  const int k0 = blockIdx.y * kper, k1 = k0 + kper < nk ? k0 + kper : nk;
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
  // scales: wavefront w loads the dwords that hold a k-tile's scales for 64 of the tile's rows, A's and then B's
  const bool sA = 64 * w < BM;
  const int srow = 64 * w + lane - (sA ? 0 : BM);
  const int sm = sA ? m0 : n0, sshift = sA ? g.shift_a : g.shift_b, sfirst = sm >> sshift;
  const int64_t slds = sA ? g.ldsa : g.ldsb;
  const int slast = ((sm + (sA ? ra : rb) - 1) >> sshift) - sfirst;
  const __amdgpu_buffer_rsrc_t rsrcS = rsrc_of((sA ? g.sa : g.sb) + sfirst * slds, slast * slds + ((nk + 3) & ~3));
  const uint32_t soff = srow < (sA ? ra : rb) && srow >= 0 ? (uint32_t)((((sm + srow) >> sshift) - sfirst) * slds) : kOutOfRange;

  typedef __attribute__((address_space(3))) void* lds_ptr_t;
  const int lds_wave = __builtin_amdgcn_readfirstlane(w * 1024), lds_scale = __builtin_amdgcn_readfirstlane(DATA + w * 256);
  auto load = [&](int kt, int stage) {
    unsigned char* const st = smem + stage * STAGE;
    const bool in = kt < k1, in_k = in && kt * 128 + chunk * 16 < Kr;
    const uint32_t koff = (uint32_t)kt * 128u;
#pragma unroll
    for (int i = 0; i < LA + LB; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(i < LA ? rsrcA : rsrcB, (lds_ptr_t)(st + lds_wave + i * 4096), 16,
                                               in_k && voff[i] != kOutOfRange ? voff[i] + koff : kOutOfRange, 0, 0, 0);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrcS, (lds_ptr_t)(st + lds_scale), 4,
                                             in && soff != kOutOfRange ? soff + (uint32_t)(kt & ~3) : kOutOfRange, 0, 0, 0);
  };
  const uint32_t fragA = (uint32_t)((wm * (BM / 2) + lrow) * 128), fragB = (uint32_t)(A_BYTES + (wn * (BN / 2) + lrow) * 128);
  const uint32_t x0 = (uint32_t)((lgrp ^ ((lane >> 1) & 7)) << 4), x1 = x0 ^ 64;
  const uint32_t scaleA = (uint32_t)(DATA + (wm * (BM / 2) + lrow) * 4), scaleB = (uint32_t)(DATA + (BM + wn * (BN / 2) + lrow) * 4);

  f32x4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

#pragma unroll
  for (int s = 0; s < NS - 1; ++s) load(k0 + s, s);
  for (int kt = k0; kt < k1; ++kt) {
    // this wavefront's part of k-tile kt has landed and its reads of the last one are done; behind the barrier, everybody's
    __builtin_amdgcn_s_waitcnt(SLP_VMCNT_LGKM0((NS - 2) * NLD));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int step = kt - k0;
    load(kt + NS - 1, (step + NS - 1) % NS);
    const unsigned char* const st = smem + step % NS * STAGE;
    Fragment<EXACT> a[MI], b[NI];
    auto fragment = [&](uint32_t at) {
      const u32x4 lo = *(const u32x4*)(st + at + x0), hi = *(const u32x4*)(st + at + x1);
      return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    };
#pragma unroll
    for (int j = 0; j < NI; ++j) b[j].set(fragment(fragB + j * 2048), st[scaleB + j * 64 + (kt & 3)]);
#pragma unroll
    for (int i = 0; i < MI; ++i) a[i].set(fragment(fragA + i * 2048), st[scaleA + i * 64 + (kt & 3)]);
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = mma(b[j], a[i], acc[i][j]);
  }
  __builtin_amdgcn_s_waitcnt(SLP_VMCNT(0));      // no load into LDS may outlive the workgroup

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

template <int BM, int BN, int NS, bool EXACT>
hipError_t configure_tile() {
  static std::once_flag once;
  static hipError_t result = hipSuccess;
  std::call_once(once, [] {
    result = hipFuncSetAttribute((const void*)product_tile_kernel<BM, BN, NS, EXACT>, hipFuncAttributeMaxDynamicSharedMemorySize, NS * ((BM + BN) * 128 + 1024));
  });
  return result;
}

// Parts of the contraction: as many as give each of the 256 compute units a workgroup, of 4 k-tiles at least.
int parts_of(int M, int N, int K, int BM, int BN) {
  const int64_t tiles = (int64_t)((M + BM - 1) / BM) * ((N + BN - 1) / BN);
  const int nk = (K + 127) / 128;
  int64_t parts = tiles >= 192 ? 1 : 256 / tiles;
  if (parts > nk / 4) parts = nk / 4;
  return parts < 1 ? 1 : (int)parts;
}

template <int BM, int BN, int NS, bool EXACT>
hipError_t launch_tile(const ProductArgs& g, hipStream_t s) {
  hipError_t e = configure_tile<BM, BN, NS, EXACT>();
  if (e != hipSuccess) return e;
  const unsigned tiles = (unsigned)(((g.M + BM - 1) / BM) * ((g.N + BN - 1) / BN));
  const int nk = (g.K + 127) / 128, wanted = parts_of(g.M, g.N, g.K, BM, BN);
  const int kper = nk > wanted ? (nk + wanted - 1) / wanted : 1, parts = nk > 1 ? (nk + kper - 1) / kper : 1;
  hipLaunchKernelGGL((product_tile_kernel<BM, BN, NS, EXACT>), dim3(tiles, parts), dim3(256), NS * ((BM + BN) * 128 + 1024), s, g, kper);
  e = hipGetLastError();
  if (e != hipSuccess || parts == 1) return e;
  const int64_t quads = (int64_t)g.M * ((g.N + 3) / 4);
  join_kernel<<<(unsigned)((quads + 255) / 256), 256, 0, s>>>(g, parts);
  return hipGetLastError();
}

bool wide_tiles(int M, int N) { return (int64_t)((M + 127) / 128) * ((N + 127) / 128) >= 192; }

}  // namespace

size_t product_floats(int M, int N, int K) {
  const int t = wide_tiles(M, N) ? 128 : 64, parts = parts_of(M, N, K, t, t);
  return parts > 1 ? (size_t)parts * M * ((N + 3) & ~3) : 0;
}

hipError_t launch_product(const ProductArgs& g, hipStream_t s) {
  const bool wide = wide_tiles(g.M, g.N);
  if (g.out_dtype == 0) return wide ? launch_tile<128, 128, 2, true>(g, s) : launch_tile<64, 64, 4, true>(g, s);
  return wide ? launch_tile<128, 128, 2, false>(g, s) : launch_tile<64, 64, 4, false>(g, s);
}

hipError_t product_configure_all() {
  hipError_t e = configure_tile<128, 128, 2, false>();
  if (e == hipSuccess) e = configure_tile<64, 64, 4, false>();
  if (e == hipSuccess) e = configure_tile<128, 128, 2, true>();
  return e == hipSuccess ? configure_tile<64, 64, 4, true>() : e;
}

}  // namespace slp
