// Matrix products of the losses over the classes of a linear layer: logits that never go to memory as a whole, and what their gradient is multiplied with.
//
//   STATS  z = (x W^T + b) / T, tile by tile; a row's largest z and sum of exp(z - largest) over each wavefront's columns leave the chip, nothing else
//   PROB   z again, p = softmax(z) for a piece of the classes, row-major and transposed
//   OUT    dx = P W (a long contraction, split over the chip where there are few tiles), dW = P^T x
//
// Float32 operands go through the bf16 matrix unit, which does 16 times the float32 one's work: each value is the sum of three bf16 values (8 bits of its 24
// each, exact above 2^-110), and of the nine products of two values' parts the six largest are added in float32; the three left out are below 2^-26 of the product,
// where float32 itself rounds each step by 2^-24.
#include "class_loss.h"
#include "eightbit_device.h"
#include "gemm_launch.h"
#include "long_tile.h"

namespace slp {
namespace {

constexpr int kXcds = 8;
constexpr uint32_t kOutOfRange = 0x80000000u;     // byte offset past the end of every tile
constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_of(const void* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00020000);
}

// What a lane feeds the matrix unit with from 32 bytes of a row, two of the 16-byte pieces of its 128: 2 x 8 bf16, or 8 float32 in three parts.
template <typename T> struct Fragment;
template <> struct Fragment<bf16> {
  bf16x8 v[2];
  __device__ __forceinline__ void set(const u32x4& lo, const u32x4& hi) {
    v[0] = __builtin_bit_cast(bf16x8, lo);
    v[1] = __builtin_bit_cast(bf16x8, hi);
  }
};
template <> struct Fragment<float> {
  bf16x8 v[3];
  __device__ __forceinline__ void set(const u32x4& lo, const u32x4& hi) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t bits = e < 4 ? lo[e & 3] : hi[e & 3];
      const float x = __builtin_bit_cast(float, bits);
      v[0][e] = (bf16)x;
      const float r = x - (float)v[0][e];
      v[1][e] = (bf16)r;
      v[2][e] = (bf16)(r - (float)v[1][e]);
    }
  }
};
__device__ __forceinline__ f32x4 mfma(const bf16x8& b, const bf16x8& a, const f32x4& acc) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, a, acc, 0, 0, 0); }
// (operands in the order B, A: a lane then holds 4 consecutive columns of one row of the output)
__device__ __forceinline__ f32x4 mma(const Fragment<bf16>& b, const Fragment<bf16>& a, f32x4 acc) {
  acc = mfma(b.v[0], a.v[0], acc);
  return mfma(b.v[1], a.v[1], acc);
}
__device__ __forceinline__ f32x4 mma(const Fragment<float>& b, const Fragment<float>& a, f32x4 acc) {
  acc = mfma(b.v[2], a.v[0], acc);
  acc = mfma(b.v[0], a.v[2], acc);
  acc = mfma(b.v[1], a.v[1], acc);
  acc = mfma(b.v[1], a.v[0], acc);
  acc = mfma(b.v[0], a.v[1], acc);
  return mfma(b.v[0], a.v[0], acc);
}

// 4x4 transpose across the 4 lanes of a quad: on return, lane i holds in v[j] what lane j held in v[i].
__device__ __forceinline__ float quad_swap(float x, bool by_two) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  return __builtin_bit_cast(float, by_two ? dpp<kSwap2>(u) : dpp<kSwap1>(u));
}
__device__ __forceinline__ void quad_transpose(f32x4& v, int lane) {
  const bool b0 = lane & 1, b1 = lane & 2;
  float r;
  r = quad_swap(b0 ? v[0] : v[1], false); if (b0) v[0] = r; else v[1] = r;
  r = quad_swap(b0 ? v[2] : v[3], false); if (b0) v[2] = r; else v[3] = r;
  r = quad_swap(b1 ? v[0] : v[2], true);  if (b1) v[0] = r; else v[2] = r;
  r = quad_swap(b1 ? v[1] : v[3], true);  if (b1) v[1] = r; else v[3] = r;
}

// Four consecutive elements, rounded to the type; `left` of them exist.
__device__ __forceinline__ void store4(bf16* out, int left, const f32x4& v) {
  const bf16x4 o = {(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
  if (left >= 4) ((AnyBf16x4*)out)->v = o;
  else
    for (int e = 0; e < left; ++e) out[e] = o[e];
}
__device__ __forceinline__ void store4(float* out, int left, const f32x4& v) {
  if (left >= 4) ((AnyF32x4*)out)->v = v;
  else
    for (int e = 0; e < left; ++e) out[e] = v[e];
}

// Over the lanes l, l ^ 16, l ^ 32 and l ^ 48.
__device__ __forceinline__ float fmax_of_rows(float x) {
  uint32_t u = __builtin_bit_cast(uint32_t, x);
  u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(u, u, false, false));
  uint32_t a = r[0], b = r[1];
  u = __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
  r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(u, u, false, false));
  a = r[0];
  b = r[1];
  return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

// The tail of a wavefront's (16 MI) x (16 NI) sums at row m0, column n0: lane l holds in acc[i][j] the columns n0 + 16 j + 4 (l / 16) .. + 3 of row
// m0 + 16 i + l % 16.
template <typename T, int KIND, int MI, int NI>
__device__ __forceinline__ void finish(const ClassProduct& g, f32x4 (&acc)[MI][NI], int m0, int n0, int lane) {
  const int lgrp = lane >> 4, lrow = lane & 15;
  if constexpr (KIND == PRODUCT_OUT) {
    if (g.work) {
      const int64_t ldw = (g.N + 3) & ~3;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int n = n0 + 16 * j + 4 * lgrp;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
          const int m = m0 + 16 * i + lrow;
          if (m < g.M && n < g.N) {
            f32x4* const to = (f32x4*)(g.work + ((int64_t)blockIdx.y * g.M + m) * ldw + n);
            *to = g.add ? *to + acc[i][j] : acc[i][j];
          }
        }
      }
    } else {
      const float alpha = *g.alpha;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int n = n0 + 16 * j + 4 * lgrp;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
          const int m = m0 + 16 * i + lrow;
          if (m < g.M && n < g.N) {
            const int64_t at = (int64_t)m * g.ldo + n;
            if (g.out_dtype == 1) store4((bf16*)g.out + at, g.N - n, acc[i][j] * alpha);
            else store4((float*)g.out + at, g.N - n, acc[i][j] * alpha);
          }
        }
      }
    }
  } else {
    // logits; those past the last class are -infinity
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int n = n0 + 16 * j + 4 * lgrp;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float bias = g.bias && n + e < g.N ? g.bias[n + e] : 0.0f;
#pragma unroll
        for (int i = 0; i < MI; ++i) acc[i][j][e] = n + e < g.N ? (acc[i][j][e] + bias) * g.per_t : -INFINITY;
      }
    }
    if constexpr (KIND == PRODUCT_STATS) {
      const int span = n0 / (16 * NI);
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        float most = -INFINITY;
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) most = fmaxf(most, acc[i][j][e]);
        most = fmax_of_rows(most);
        const float from = most == -INFINITY ? 0.0f : most;
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f((acc[i][j][e] - from) * kLog2e);
        sum = sum_of_rows(sum);
        const int m = m0 + 16 * i + lrow;
        if (lgrp == 0 && m < g.M) g.stats[(int64_t)span * g.M + m] = float2{most, sum};
      }
    } else {
      const int last_n = (g.N + 7) & ~7, last_m = (g.M + 7) & ~7;
      float2 norm[MI];
      int label[MI];
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const int m = m0 + 16 * i + lrow;
        norm[i] = m < g.M ? g.norm[m] : float2{INFINITY, 0.0f};
        label[i] = g.labels && m < g.M ? g.labels[m] - g.label0 : -1;
      }
      const int part = m0 / (16 * MI);
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int n = n0 + 16 * j + 4 * lgrp;
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < MI; ++i) {
          const int m = m0 + 16 * i + lrow;
          f32x4 p;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[e] = __builtin_amdgcn_exp2f((acc[i][j][e] - norm[i].x) * kLog2e) * norm[i].y;
            if (norm[i].x == INFINITY || n + e == label[i] || n + e >= g.N) p[e] = 0.0f;       // (also where the row holds NaN)
          }
          sum += p;
          if (m < g.M && n < last_n) {
            T* const to = (T*)g.p + (int64_t)m * g.ldp + n;
            store4(to, 4, p);
          }
          if (g.pt) {
            quad_transpose(p, lane);      // now 4 rows of column n + lane % 4
            const int c = n + (lane & 3), r = m - (lane & 3);
            if (c < g.N && r < last_m) store4((T*)g.pt + (int64_t)c * g.ldpt + r, 4, p);
          }
        }
        if (g.sums) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float all = sum_of_16(sum[e]);
            if (lrow == 0 && n + e < g.N) g.sums[(int64_t)part * g.N + n + e] = all;
          }
        }
      }
    }
  }
}

// workgroup -> tile: consecutive workgroups go round the XCDs; each XCD walks a contiguous run of tiles, 8 tile rows high.
__device__ __forceinline__ void tile_of(int tilesM, int tilesN, int& tm, int& tn) {
  const int total = tilesM * tilesN, pid = blockIdx.x, xcd = pid % kXcds, q = pid / kXcds, base = total / kXcds, rem = total % kXcds;
  const int tid = xcd * base + (xcd < rem ? xcd : rem) + q;
  constexpr int kGroup = 8;
  const int width = kGroup * tilesN, first = tid / width * kGroup, rows = tilesM - first < kGroup ? tilesM - first : kGroup;
  tm = first + tid % width % rows;
  tn = tid % width / rows;
}

// BM x BN tile, 4 wavefronts in a 2 x 2 grid, NS LDS stages of a k-tile of 128 bytes each, one barrier a k-tile.  blockIdx.y: part of the contraction, kper
// k-tiles long.
template <typename T, int KIND, int BM, int BN, int NS>
__global__ __launch_bounds__(256) void class_tile_kernel(const ClassProduct g, int kper) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int ES = sizeof(T), BK = 128 / ES, CH = 16 / ES;
  constexpr int A_BYTES = BM * 128, STAGE = (BM + BN) * 128;
  constexpr int LA = BM / 32, LB = BN / 32, NLD = LA + LB, MI = BM / 32, NI = BN / 32;
  int tm, tn;
  tile_of((g.M + BM - 1) / BM, (g.N + BN - 1) / BN, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, wm = w & 1, wn = w >> 1, lgrp = lane >> 4, lrow = lane & 15;
  const int64_t lda = g.lda * ES, ldb = g.ldb * ES;
  const int nk = (g.K + BK - 1) / BK, Kr = (g.K + CH - 1) / CH * 16;       // bytes of a row, to the end of its last 16
  const int k0 = blockIdx.y * kper, k1 = k0 + kper < nk ? k0 + kper : nk;
  const int ra = g.M - m0 < BM ? g.M - m0 : BM, rb = g.N - n0 < BN ? g.N - n0 : BN;        // rows of the tile that exist
  const __amdgpu_buffer_rsrc_t rsrcA = rsrc_of((const char*)g.a + (int64_t)m0 * lda, (ra - 1) * lda + Kr);
  const __amdgpu_buffer_rsrc_t rsrcB = rsrc_of((const char*)g.b + (int64_t)n0 * ldb, (rb - 1) * ldb + Kr);
  // a load of the workgroup fills 32 rows, lane l of wavefront w the 16-byte piece l % 8 of row 8 w + l / 8; piece c of a row is chunk
  // c ^ (row / 2 mod 8), which spreads the 16 rows of a fragment over all LDS banks
  const int prow = w * 8 + (lane >> 3), chunk = (lane & 7) ^ ((prow >> 1) & 7);
  uint32_t voff[NLD];
#pragma unroll
  for (int i = 0; i < LA; ++i) voff[i] = prow + 32 * i < ra ? (uint32_t)((prow + 32 * i) * lda + chunk * 16) : kOutOfRange;
#pragma unroll
  for (int i = 0; i < LB; ++i) voff[LA + i] = prow + 32 * i < rb ? (uint32_t)((prow + 32 * i) * ldb + chunk * 16) : kOutOfRange;
  typedef __attribute__((address_space(3))) void* lds_ptr_t;
  const int lds_wave = __builtin_amdgcn_readfirstlane(w * 1024);
  auto load = [&](int kt, int stage) {
    unsigned char* const st = smem + stage * STAGE;
    const bool in = kt < k1 && kt * 128 + chunk * 16 < Kr;
    const uint32_t koff = (uint32_t)kt * 128u;
#pragma unroll
    for (int i = 0; i < NLD; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(i < LA ? rsrcA : rsrcB, (lds_ptr_t)(st + lds_wave + i * 4096), 16,
                                               in && voff[i] != kOutOfRange ? voff[i] + koff : kOutOfRange, 0, 0, 0);
  };
  const uint32_t fragA = (uint32_t)((wm * (BM / 2) + lrow) * 128), fragB = (uint32_t)(A_BYTES + (wn * (BN / 2) + lrow) * 128);
  const uint32_t x0 = (uint32_t)((lgrp ^ ((lane >> 1) & 7)) << 4), x1 = x0 ^ 64;
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
    load(kt + NS - 1, (kt - k0 + NS - 1) % NS);
    const unsigned char* const st = smem + (kt - k0) % NS * STAGE;
    Fragment<T> a[MI], b[NI];
#pragma unroll
    for (int j = 0; j < NI; ++j) b[j].set(*(const u32x4*)(st + fragB + j * 2048 + x0), *(const u32x4*)(st + fragB + j * 2048 + x1));
#pragma unroll
    for (int i = 0; i < MI; ++i) a[i].set(*(const u32x4*)(st + fragA + i * 2048 + x0), *(const u32x4*)(st + fragA + i * 2048 + x1));
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = mma(b[j], a[i], acc[i][j]);
  }
  __builtin_amdgcn_s_waitcnt(SLP_VMCNT(0));      // no load into LDS may outlive the workgroup
  finish<T, KIND, MI, NI>(g, acc, m0 + wm * (BM / 2), n0 + wn * (BN / 2), lane);
#endif
}

// Large bf16 products (long_tile.h).  What the epilogues of the tiles above do, with the accumulators taken out of the AGPRs a block at a time, and stores of whole
// row segments: a wavefront stages its 128 x 128 outputs in a 32 KB of the stages that is its own, rows of 256 bytes whose 16-byte piece c sits at c ^ swz(row), and takes
// them out row by row and, through transposing LDS reads (a group of 16 lanes reads 4 rows of 16 columns, lane l gets the 4 values of column l), column by column.
// 16 rows in a row lie on 16 pieces, the 8 rows that half a wavefront reads transposed on disjoint ones.
template <int KIND>
__global__ __launch_bounds__(256) void class_long_kernel(const ClassProduct g, int kper) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef __attribute__((ext_vector_type(4))) short i16x4;
  typedef __attribute__((address_space(3))) i16x4* lds_i16x4;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  int tm, tn;
  big_tile(g.M, g.N, tm, tn);
  const int m0 = tm * 256, n0 = tn * 256;
  f32x4 acc[8][8];
  {
    const int64_t lda = g.lda * 2, ldb = g.ldb * 2, from = (int64_t)blockIdx.y * kper * 128, all = (int64_t)g.K * 2 - from, part = (int64_t)kper * 128;
    const int K = all <= 0 ? 0 : (int)(all < part ? all : part);
    const int64_t at = all <= 0 ? 0 : from;
    long_tile<f32x4, false>(acc, smem, (const char*)g.a + m0 * lda + at, (const char*)g.b + n0 * ldb + at, lda, ldb, g.M - m0 < 256 ? g.M - m0 : 256, g.N - n0 < 256 ? g.N - n0 : 256, K);
  }
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, wm = w & 1, wn = w >> 1, lgrp = lane >> 4, lrow = lane & 15;
  const int rowW = m0 + wm * 128, colW = n0 + wn * 128;
  if constexpr (KIND == PRODUCT_STATS) {
    // z log2(e), so that the exponentials take one addition
    f32x4 bias[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = colW + 16 * j + 4 * lgrp + e;
        bias[j][e] = n >= g.N ? -INFINITY : g.bias ? g.bias[n] : 0.0f;
      }
    const int span = colW / 128;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      f32x4 z[8];
      float most = -INFINITY;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        asm volatile("" : "+a"(acc[i][j]));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          z[j][e] = (acc[i][j][e] + bias[j][e]) * g.per_t;
          most = fmaxf(most, z[j][e]);
        }
      }
      most = fmax_of_rows(most);
      const float from = most == -INFINITY ? 0.0f : most;
      float sum = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f((z[j][e] - from) * kLog2e);
      sum = sum_of_rows(sum);
      const int m = rowW + 16 * i + lrow;
      if (lgrp == 0 && m < g.M) g.stats[(int64_t)span * g.M + m] = float2{most, sum};
      __builtin_amdgcn_sched_barrier(0);
    }
    return;
  }
  auto swz = [](int r) { return ((r & 3) << 1) | (r & 8) | ((r >> 2) & 1); };
  __syncthreads();                       // nobody reads the stages any more
  unsigned char* const st = smem + w * 32768;
  unsigned char* const wbase = st + lrow * 256 + (lgrp & 1) * 8;
  const int wsw = (lgrp >> 1) ^ swz(lrow);
  auto stage = [&](int i, int j, const f32x4& v) {
    const bf16x4 o = {(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
    *(u32x2*)(wbase + i * 4096 + ((wsw ^ (2 * j)) << 4)) = __builtin_bit_cast(u32x2, o);
  };
  // 16-byte pieces of whole rows, 8 at a time: their LDS reads are under way together
  auto rows_out = [&](auto put) {
    const int r0 = lane >> 4, c = lane & 15;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      u32x4 val[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int r = (8 * b + q) * 4 + r0;
        val[q] = *(const u32x4*)(st + r * 256 + ((c ^ swz(r & 15)) << 4));
      }
#pragma unroll
      for (int q = 0; q < 8; ++q) put((8 * b + q) * 4 + r0, c * 8, val[q]);
    }
  };
  if constexpr (KIND == PRODUCT_OUT) {
    const float alpha = g.work ? 1.0f : *g.alpha;
    if (g.work || g.out_dtype == 0) {    // float32, straight from the accumulators: 64-byte segments
      const int64_t ld = g.work ? (g.N + 3) & ~3 : g.ldo;
      float* const out = g.work ? g.work + (int64_t)blockIdx.y * g.M * ld : (float*)g.out;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int n = colW + 16 * j + 4 * lgrp;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          asm volatile("" : "+a"(acc[i][j]));
          const int m = rowW + 16 * i + lrow;
          if (m < g.M && n < g.N) {
            float* const to = out + m * ld + n;
            f32x4 v = acc[i][j] * alpha;
            if (g.work) {
              if (g.add) v += *(const f32x4*)to;
              *(f32x4*)to = v;
            } else {
              store4(to, g.N - n, v);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        asm volatile("" : "+a"(acc[i][j]));
        stage(i, j, acc[i][j] * alpha);
        __builtin_amdgcn_sched_barrier(0);
      }
    rows_out([&](int r, int c, const u32x4& v) {
      const int m = rowW + r, n = colW + c;
      if (m < g.M && n < g.N) {
        bf16* const to = (bf16*)g.out + m * g.ldo + n;
        const bf16x8 o = __builtin_bit_cast(bf16x8, v);
        if (n + 8 <= g.N) ((AnyBf16x8*)to)->v = o;
        else
          for (int e = 0; e < g.N - n; ++e) to[e] = o[e];
      }
    });
  } else if constexpr (KIND == PRODUCT_PROB) {
    float2 norm[8];
    int label[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int m = rowW + 16 * i + lrow;
      norm[i] = m < g.M ? g.norm[m] : float2{INFINITY, 0.0f};
      label[i] = g.labels && m < g.M ? g.labels[m] - g.label0 : -1;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int n = colW + 16 * j + 4 * lgrp;
      f32x4 bias, sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int e = 0; e < 4; ++e) bias[e] = n + e >= g.N ? -INFINITY : g.bias ? g.bias[n + e] : 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        asm volatile("" : "+a"(acc[i][j]));
        f32x4 p;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float z = (acc[i][j][e] + bias[e]) * g.per_t;
          p[e] = __builtin_amdgcn_exp2f((z - norm[i].x) * kLog2e) * norm[i].y;
          if (norm[i].x == INFINITY || n + e == label[i] || n + e >= g.N) p[e] = 0.0f;       // (also where the row holds NaN)
        }
        sum += p;
        stage(i, j, p);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (g.sums) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float all = sum_of_16(sum[e]);
          if (lrow == 0 && n + e < g.N) g.sums[(int64_t)(rowW / 128) * g.N + n + e] = all;
        }
      }
    }
    rows_out([&](int r, int c, const u32x4& v) {
      if (rowW + r < g.M && colW + c < g.N) *(u32x4*)((bf16*)g.p + (int64_t)(rowW + r) * g.ldp + colW + c) = v;
    });
    if (g.pt) {
      const int gq = lane >> 4, jj = lane & 15, r0 = gq * 8 + (jj >> 2);        // staged row of the first of the two reads
      const uint32_t base = (uint32_t)(r0 * 256 + ((((jj & 3) >> 1) ^ swz(r0 & 15)) << 4) + (jj & 1) * 8);
#pragma unroll
      for (int b = 0; b < 8; b += 2) {
        u32x2 val[8][2];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const uint32_t o1 = (base ^ ((b + q / 4) << 5)) + q % 4 * 8192;
          val[q][0] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(st + o1)));
          val[q][1] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(st + ((o1 ^ 16) + 1024))));
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int n = colW + jj + (b + q / 4) * 16, m = rowW + gq * 8 + q % 4 * 32;
          if (n < g.N && m < g.M) *(u32x4*)((bf16*)g.pt + (int64_t)n * g.ldpt + m) = u32x4{val[q][0][0], val[q][0][1], val[q][1][0], val[q][1][1]};
        }
      }
    }
  }
#endif
}

// ---- host side -------------------------------------------------------------------------------
int64_t tiles_of(int M, int N, int BM, int BN) { return (int64_t)((M + BM - 1) / BM) * ((N + BN - 1) / BN); }

enum Shape { kLong, k128, k64 };
Shape shape_of(int dtype, int M, int N) {
  if (dtype == 1 && tiles_of(M, N, 256, 256) >= 200) return kLong;
  return tiles_of(M, N, 128, 128) >= 200 ? k128 : k64;
}
// Rows, or columns, of a wavefront's part of a tile.
int span_of(Shape s) { return s == kLong ? 128 : s == k128 ? 64 : 32; }

template <typename T, int KIND, int BM, int BN, int NS>
hipError_t launch_tile(const ClassProduct& g, hipStream_t s) {
  constexpr int smem = NS * (BM + BN) * 128;
  static std::atomic<uint64_t> done{0};
  hipError_t e = allow_lds((const void*)class_tile_kernel<T, KIND, BM, BN, NS>, smem, done);
  if (e != hipSuccess) return e;
  constexpr int BK = 128 / (int)sizeof(T);
  const int nk = (g.K + BK - 1) / BK, parts = g.work ? g.parts : 1, kper = (nk + parts - 1) / parts;
  hipLaunchKernelGGL((class_tile_kernel<T, KIND, BM, BN, NS>), dim3((unsigned)tiles_of(g.M, g.N, BM, BN), parts), dim3(256), smem, s, g, kper);
  return hipGetLastError();
}
template <int KIND>
hipError_t launch_long(const ClassProduct& g, hipStream_t s) {
  static std::atomic<uint64_t> done{0};
  const hipError_t e = allow_lds((const void*)class_long_kernel<KIND>, kLongSmem, done);
  if (e != hipSuccess) return e;
  const int nk = (g.K + 63) / 64, parts = g.work ? g.parts : 1, kper = (nk + parts - 1) / parts;
  class_long_kernel<KIND><<<dim3((unsigned)tiles_of(g.M, g.N, 256, 256), parts), 256, kLongSmem, s>>>(g, kper);
  return hipGetLastError();
}
template <typename T, int KIND>
hipError_t launch_kind(int dtype, const ClassProduct& g, hipStream_t s) {
  switch (shape_of(dtype, g.M, g.N)) {
    case kLong:
      if constexpr (sizeof(T) == 2) return launch_long<KIND>(g, s);
    case k128: return launch_tile<T, KIND, 128, 128, 2>(g, s);
    default: return launch_tile<T, KIND, 64, 64, 2>(g, s);
  }
}
template <typename T>
hipError_t launch_type(int dtype, int kind, const ClassProduct& g, hipStream_t s) {
  switch (kind) {
    case PRODUCT_STATS: return launch_kind<T, PRODUCT_STATS>(dtype, g, s);
    case PRODUCT_PROB: return launch_kind<T, PRODUCT_PROB>(dtype, g, s);
    default: return launch_kind<T, PRODUCT_OUT>(dtype, g, s);
  }
}

}  // namespace

int stats_spans(int dtype, int M, int N) {
  const int w = span_of(shape_of(dtype, M, N));
  return (N + 2 * w - 1) / (2 * w) * 2;
}
int sum_parts(int dtype, int M, int N) {
  const int w = span_of(shape_of(dtype, M, N));
  return (M + 2 * w - 1) / (2 * w) * 2;
}

hipError_t launch_class_product(int dtype, int kind, const ClassProduct& g, hipStream_t s) {
  const int64_t es = dtype == 1 ? 2 : 4;
  // a tile's rows are addressed with 32-bit offsets
  if (g.M <= 0 || g.N <= 0 || g.K <= 0 || 256 * g.lda * es >= 0x7FFFFF00 || 256 * g.ldb * es >= 0x7FFFFF00) return hipErrorInvalidValue;
  if ((((uintptr_t)g.a | (uintptr_t)g.b) & 15) || g.lda * es % 16 || g.ldb * es % 16) return hipErrorInvalidValue;
  return dtype == 1 ? launch_type<bf16>(dtype, kind, g, s) : launch_type<float>(dtype, kind, g, s);
}

}  // namespace slp
