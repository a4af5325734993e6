// Matrix products of the losses over the classes of a linear layer: logits that never go to memory as a whole, and what their gradient is multiplied with.
//
//   STATS  z = (x W^T + b) / T, tile by tile; a row's largest z and sum of exp(z - largest) over each wavefront's columns leave the chip, and z where it is kept
//   PROB   z again, p = softmax(z) for a piece of the classes, row-major and transposed
//   DX     P W, a contraction over the piece's classes, split over the chip where there are few tiles
//   DW     P^T x, over the rows
// W lies in DX, and both operands in DW, with a row for each step of the contraction: their tiles are read transposed from LDS, so that nothing has to be
// written twice.
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
  if constexpr (KIND >= PRODUCT_DX) {
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
        if (g.z && m < g.M) {
#pragma unroll
          for (int j = 0; j < NI; ++j) {
            const int n = n0 + 16 * j + 4 * lgrp;
            if (n < g.zcols) *(f32x4*)(g.z + (int64_t)m * g.ldz + n) = acc[i][j];
          }
        }
        if (lgrp == 0 && m < g.M) g.stats[(int64_t)span * g.M + m] = float2{most, sum};
      }
    } else {
      const int last_n = (g.N + 7) & ~7;
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

// One operand of a tile in LDS: ROWS rows (columns of a matrix that lies the other way) by 128 bytes of the contraction.
//   rows by contraction: a load of the workgroup fills 32 rows, lane l of wavefront w the 16-byte piece l % 8 of row 8 w + l / 8; piece c of a row sits at c ^ (row / 2
//   mod 8), which spreads the 16 rows of a fragment over all LDS banks
//   KM, the other way: BK rows of ROWS columns; piece c of row k sits at c ^ key(k), so that what half a wavefront reads of 8 rows (bf16, transposing reads) or a wavefront of 4
//   (float32) lies on all banks.
template <typename T, int ROWS, bool KM>
struct Side {
  static constexpr int ES = sizeof(T), BK = 128 / ES, LOADS = ROWS / 32, PIECES = ROWS * ES / 16;     // loads of a k-tile; KM: pieces of a row
  __amdgpu_buffer_rsrc_t rsrc;
  uint32_t voff[LOADS];
  uint32_t step;            // bytes from a k-tile to the next
  int k[LOADS], K;          // KM: rows of the loads in a k-tile, the contraction's length; otherwise k[0]: first byte of the piece, K: bytes
  static __device__ __forceinline__ int key(int k) {
    if constexpr (ES == 4) return ((k >> 2) & 3) << 2;
    else if constexpr (PIECES >= 16) return ((k & 3) | ((k >> 1) & 4)) << 1;
    else return (((k >> 1) & 1) | ((k >> 2) & 2)) << 1;
  }
  // rows (columns) [first, first + n) exist, n <= ROWS
  __device__ __forceinline__ void init(const void* p, int64_t ld, int first, int n, int K_, int t) {
    const int64_t bytes = ld * ES;
    if constexpr (!KM) {
      const int prow = t >> 3, chunk = (t & 7) ^ ((prow >> 1) & 7);
      K = (K_ * ES + 15) & ~15;
      rsrc = rsrc_of((const char*)p + first * bytes, (n - 1) * bytes + K);
      k[0] = chunk * 16;
      step = 128;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) voff[i] = prow + 32 * i < n ? (uint32_t)((prow + 32 * i) * bytes + chunk * 16) : kOutOfRange;
    } else {
      const int width = (n * ES + 15) & ~15;
      K = K_;
      rsrc = rsrc_of((const char*)p + (int64_t)first * ES, (K - 1) * bytes + width);
      step = (uint32_t)(BK * bytes);
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        k[i] = (t + 256 * i) / PIECES;
        const int c = (t % PIECES) ^ key(k[i]);
        voff[i] = c * 16 < width ? (uint32_t)(k[i] * bytes + c * 16) : kOutOfRange;
      }
    }
  }
  __device__ __forceinline__ void load(unsigned char* to, int kt, bool in) const {
    typedef __attribute__((address_space(3))) void* lds_ptr_t;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const bool exists = in && voff[i] != kOutOfRange && (KM ? kt * BK + k[i] < K : kt * 128 + k[0] < K);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_ptr_t)(to + i * 4096), 16, exists ? voff[i] + (uint32_t)kt * step : kOutOfRange, 0, 0, 0);
    }
  }
  // 32 bytes of the contraction for row (column) r0 + lane % 16, those that the other operand's fragment takes
  __device__ __forceinline__ Fragment<T> fragment(const unsigned char* st, int r0, int lane) const {
    const int lgrp = lane >> 4, lrow = lane & 15;
    Fragment<T> f;
    if constexpr (!KM) {
      const unsigned char* const row = st + (r0 + lrow) * 128;
      const int x0 = (lgrp ^ ((lane >> 1) & 7)) << 4;
      f.set(*(const u32x4*)(row + x0), *(const u32x4*)(row + (x0 ^ 64)));
    } else if constexpr (ES == 2) {
      typedef __attribute__((ext_vector_type(4))) short i16x4;
      typedef __attribute__((address_space(3))) i16x4* lds_i16x4;
      const int row = lgrp * 8 + (lrow >> 2), c = (r0 >> 3) + ((lrow & 3) >> 1);
      const unsigned char* const at = st + row * (ROWS * 2) + ((c ^ key(row)) << 4) + (lrow & 1) * 8;
      u32x2 v[4];
#pragma unroll
      for (int h = 0; h < 4; ++h) v[h] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(at + ((h >> 1) * 32 + (h & 1) * 4) * (ROWS * 2))));
      f.set(u32x4{v[0][0], v[0][1], v[1][0], v[1][1]}, u32x4{v[2][0], v[2][1], v[3][0], v[3][1]});
    } else {
      const int c = (r0 + lrow) >> 2;
      u32x4 v[2];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int row = (e >> 2) * 16 + lgrp * 4 + (e & 3);
        v[e >> 2][e & 3] = *(const uint32_t*)(st + row * (ROWS * 4) + ((c ^ key(row)) << 4) + (lrow & 3) * 4);
      }
      f.set(v[0], v[1]);
    }
    return f;
  }
};

// BM x BN tile, 4 wavefronts in a 2 x 2 grid, NS LDS stages of a k-tile of 128 bytes each, one barrier a k-tile.  blockIdx.y: part of the contraction, kper
// k-tiles long.
template <typename T, int KIND, int BM, int BN, int NS>
__global__ __launch_bounds__(256) void class_tile_kernel(const ClassProduct g, int kper) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  constexpr int BK = 128 / (int)sizeof(T), A_BYTES = BM * 128, STAGE = (BM + BN) * 128, NLD = (BM + BN) / 32, MI = BM / 32, NI = BN / 32;
  int tm, tn;
  tile_of((g.M + BM - 1) / BM, (g.N + BN - 1) / BN, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, wm = w & 1, wn = w >> 1;
  const int nk = (g.K + BK - 1) / BK, k0 = blockIdx.y * kper, k1 = k0 + kper < nk ? k0 + kper : nk;
  Side<T, BM, KIND == PRODUCT_DW> A;
  Side<T, BN, KIND >= PRODUCT_DX> B;
  A.init(g.a, g.lda, m0, g.M - m0 < BM ? g.M - m0 : BM, g.K, t);
  B.init(g.b, g.ldb, n0, g.N - n0 < BN ? g.N - n0 : BN, g.K, t);
  const int lds_wave = __builtin_amdgcn_readfirstlane(w * 1024);
  auto load = [&](int kt, int stage) {
    unsigned char* const st = smem + stage * STAGE + lds_wave;
    A.load(st, kt, kt < k1);
    B.load(st + A_BYTES, kt, kt < k1);
  };
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
    for (int j = 0; j < NI; ++j) b[j] = B.fragment(st + A_BYTES, wn * (BN / 2) + 16 * j, lane);
#pragma unroll
    for (int i = 0; i < MI; ++i) a[i] = A.fragment(st, wm * (BM / 2) + 16 * i, lane);
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = mma(b[j], a[i], acc[i][j]);
  }
  __builtin_amdgcn_s_waitcnt(SLP_VMCNT(0));      // no load into LDS may outlive the workgroup
  finish<T, KIND, MI, NI>(g, acc, m0 + wm * (BM / 2), n0 + wn * (BN / 2), lane);
#endif
}

// Large bf16 products (long_tile.h).  What the epilogues of the tiles above do, with the accumulators taken out of the AGPRs a block at a time; bf16 outputs leave as whole
// row segments, staged by each wavefront in a 32 KB of the stages that is its own, rows of 256 bytes whose 16-byte piece c sits at c ^ (row mod 16).
template <int KIND>
__global__ __launch_bounds__(256) void class_long_kernel(const ClassProduct g, int kper) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  int tm, tn;
  big_tile(g.M, g.N, tm, tn);
  const int m0 = tm * 256, n0 = tn * 256;
  f32x4 acc[8][8];
  {
    const int64_t lda = g.lda * 2, ldb = g.ldb * 2, from = (int64_t)blockIdx.y * kper * 128, all = (int64_t)g.K * 2 - from, part = (int64_t)kper * 128;
    const int K = all <= 0 ? 0 : (int)(all < part ? all : part);
    const int64_t at = all <= 0 ? 0 : from;
    constexpr bool KMA = KIND == PRODUCT_DW, KMB = KIND >= PRODUCT_DX;
    long_tile<f32x4, false, KMA, KMB>(acc, smem, (const char*)g.a + (KMA ? at / 2 * lda + m0 * 2 : m0 * lda + at), (const char*)g.b + (KMB ? at / 2 * ldb + n0 * 2 : n0 * ldb + at), lda, ldb, g.M - m0 < 256 ? g.M - m0 : 256, g.N - n0 < 256 ? g.N - n0 : 256, K);
  }
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, wm = w & 1, wn = w >> 1, lgrp = lane >> 4, lrow = lane & 15;
  const int rowW = m0 + wm * 128, colW = n0 + wn * 128;
  if constexpr (KIND == PRODUCT_STATS) {
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
      if (g.z && m < g.M) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int n = colW + 16 * j + 4 * lgrp;
          if (n < g.zcols) *(f32x4*)(g.z + (int64_t)m * g.ldz + n) = z[j];
        }
      }
      if (lgrp == 0 && m < g.M) g.stats[(int64_t)span * g.M + m] = float2{most, sum};
      __builtin_amdgcn_sched_barrier(0);
    }
    return;
  }
  __syncthreads();                       // nobody reads the stages any more
  unsigned char* const st = smem + w * 32768;
  unsigned char* const wbase = st + lrow * 256 + (lgrp & 1) * 8;
  const int wsw = (lgrp >> 1) ^ lrow;
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
        val[q] = *(const u32x4*)(st + r * 256 + ((c ^ (r & 15)) << 4));
      }
#pragma unroll
      for (int q = 0; q < 8; ++q) put((8 * b + q) * 4 + r0, c * 8, val[q]);
    }
  };
  if constexpr (KIND >= PRODUCT_DX) {
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
  }
#endif
}

// ---- host side -------------------------------------------------------------------------------
int64_t tiles_of(int M, int N, int BM, int BN) { return (int64_t)((M + BM - 1) / BM) * ((N + BN - 1) / BN); }

enum Shape { kLong, k128, k64 };
// parts: of the contraction, which share the chip
Shape shape_of(int dtype, int M, int N, int parts = 1) {
  if (dtype == 1 && tiles_of(M, N, 256, 256) * parts >= 200) return kLong;
  return tiles_of(M, N, 128, 128) * parts >= 200 ? k128 : k64;
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
  switch (shape_of(dtype, g.M, g.N, g.work ? g.parts : 1)) {
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
    case PRODUCT_DX: return launch_kind<T, PRODUCT_DX>(dtype, g, s);
    default: return launch_kind<T, PRODUCT_DW>(dtype, g, s);
  }
}

}  // namespace

// As many parts as make one round of the largest tiles that then have 16 k-tiles each.
int class_parts(int dtype, int M, int N, int K) {
  const int64_t nk = (K + (dtype == 1 ? 63 : 31)) / (dtype == 1 ? 64 : 32);
  auto parts = [&](int tile, int round, int least) {
    const int64_t want = round / tiles_of(M, N, tile, tile), most = nk / least;
    return (int)(want < most ? want : most);
  };
  if (dtype == 1 && tiles_of(M, N, 256, 256) * (nk / 16) >= 200) {
    const int p = parts(256, 256, 16);
    return p < 1 ? 1 : p;
  }
  const int p = tiles_of(M, N, 128, 128) * (nk / 8) >= 200 ? parts(128, 512, 8) : parts(64, 512, 4);
  return p < 1 ? 1 : p;
}

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
  // a tile's rows, or an operand that lies the other way, are addressed with 32-bit offsets
  const int64_t rows_a = kind == PRODUCT_DW ? g.K : 256, rows_b = kind >= PRODUCT_DX ? g.K : 256;
  if (g.M <= 0 || g.N <= 0 || g.K <= 0 || rows_a * g.lda * es >= 0x7FFFFF00 || rows_b * g.ldb * es >= 0x7FFFFF00) return hipErrorInvalidValue;
  if ((((uintptr_t)g.a | (uintptr_t)g.b) & 15) || g.lda * es % 16 || g.ldb * es % 16) return hipErrorInvalidValue;
  return dtype == 1 ? launch_type<bf16>(dtype, kind, g, s) : launch_type<float>(dtype, kind, g, s);
}

}  // namespace slp
