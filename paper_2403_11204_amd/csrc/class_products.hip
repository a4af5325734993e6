// Matrix products of the losses over the classes of a linear layer: logits that never go to memory as a whole, and what their gradient is multiplied with.
//
//   STATS  z = (x W^T + b) / T, tile by tile; a row's largest z and sum of exp(z - largest) over each wavefront's columns leave the chip, and z where it is kept
//   PROB   z again, p = softmax(z) for a piece of the classes whose logits are not kept
//   Z      x W^T over parts of the contraction, where there are few tiles and it is long
//   DX     P W, a contraction over the piece's classes, split over the chip where there are few tiles
//   DW     P^T x, over the rows
// P leaves PROB (or kept_prob_kernel) rounded to the operands' type, bf16 by half a step of 2^-8, as the gradient of any layer in bf16 is: in two parts it would be twice the work of
// both products.  Its common factor T scale / n, and 1 less at a row's own class, are applied in float32 around that.
// W lies in DX, and both operands in DW, with a row for each step of the contraction: their tiles are read transposed from LDS, so that nothing has to be
// written twice.
//
// Float32 operands go through the bf16 matrix unit, which does 16 times the float32 one's work: each value is the sum of three bf16 values (8 bits of its 24
// each, exact above 2^-102), and of the nine products of two values' parts the six largest are added in float32; the three left out are below 2^-26 of the product,
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

typedef __attribute__((ext_vector_type(2))) float f32x2;
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
  // (pairs: one conversion, two values back to float32 and two subtractions make the next part's)
  __device__ __forceinline__ void set(const u32x4& lo, const u32x4& hi) {
    u32x4 part[3];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f32x2 x = e < 2 ? f32x2{__builtin_bit_cast(float, (uint32_t)lo[2 * (e & 1)]), __builtin_bit_cast(float, (uint32_t)lo[2 * (e & 1) + 1])}
                      : f32x2{__builtin_bit_cast(float, (uint32_t)hi[2 * (e & 1)]), __builtin_bit_cast(float, (uint32_t)hi[2 * (e & 1) + 1])};
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        const uint32_t u = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
        part[q][e] = u;
        x[0] -= __builtin_bit_cast(float, u << 16);
        x[1] -= __builtin_bit_cast(float, u & 0xFFFF0000u);
      }
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) v[q] = __builtin_bit_cast(bf16x8, part[q]);
  }
};
// All fragments of A against all of B, a product of parts at a time: one on the same accumulator comes MI NI instructions later.  (operands in the order B, A: a lane then
// holds 4 consecutive columns of one row of the output)
template <typename T, int MI, int NI>
__device__ __forceinline__ void mma(f32x4 (&acc)[MI][NI], const Fragment<T> (&a)[MI], const Fragment<T> (&b)[NI]) {
  constexpr int N = sizeof(T) == 2 ? 2 : 6;
  constexpr int pa[6] = {0, 2, 1, 1, 0, 0}, pb[6] = {2, 0, 1, 0, 1, 0};        // (the smallest first)
#pragma unroll
  for (int q = 0; q < N; ++q)
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j].v[N == 2 ? q : pb[q]], a[i].v[N == 2 ? q : pa[q]], acc[i][j], 0, 0, 0);
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

// The softmax at a logit; 1 less where the class is the row's, exact where that is near 0.
__device__ __forceinline__ float probability(float z, float2 norm, bool label) {
  if (label) return expm1f(z - norm.x + logf(norm.y));
  return __builtin_amdgcn_exp2f((z - norm.x) * kLog2e) * norm.y;
}

// The tail of a wavefront's (16 MI) x (16 NI) sums at row m0, column n0: lane l holds in acc[i][j] the columns n0 + 16 j + 4 (l / 16) .. + 3 of row
// m0 + 16 i + l % 16.
template <typename T, int KIND, int MI, int NI>
__device__ __forceinline__ void finish(const ClassProduct& g, f32x4 (&acc)[MI][NI], int m0, int n0, int lane) {
  const int lgrp = lane >> 4, lrow = lane & 15;
  if constexpr (KIND >= PRODUCT_DX) {
    // (float32, see Side::fragments: rows that lie the other way are dealt out one by one, columns 4 NI side by side to a lane)
    constexpr bool AROUND = sizeof(T) == 4 && KIND == PRODUCT_DW, BROUND = sizeof(T) == 4 && KIND != PRODUCT_Z;
    auto row = [&](int i) { return AROUND ? m0 + MI * lrow + i : m0 + 16 * i + lrow; };
    auto col = [&](int j) { return BROUND ? n0 + 4 * NI * lgrp + 4 * j : n0 + 16 * j + 4 * lgrp; };
    // (to bf16; float32 has gone through LDS, and the bf16 of larger bf16 tiles)
    const float alpha = *g.alpha;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int n = col(j);
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const int m = row(i);
        if (m < g.M && n < g.N) store4((bf16*)g.out + (int64_t)m * g.ldo + n, g.N - n, acc[i][j] * alpha);
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
            p[e] = probability(acc[i][j][e], norm[i], n + e == label[i]);
            if (norm[i].x == INFINITY || n + e >= g.N) p[e] = 0.0f;       // (also where the row holds NaN)
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
__device__ __forceinline__ void tile_of(int pid, int tilesM, int tilesN, int& tm, int& tn) {
  const int total = tilesM * tilesN, xcd = pid % kXcds, q = pid / kXcds, base = total / kXcds, rem = total % kXcds;
  const int tid = xcd * base + (xcd < rem ? xcd : rem) + q;
  constexpr int kGroup = 8;
  const int width = kGroup * tilesN, first = tid / width * kGroup, rows = tilesM - first < kGroup ? tilesM - first : kGroup;
  tm = first + tid % width % rows;
  tn = tid % width / rows;
}

// One operand of a tile in LDS: ROWS rows (columns of a matrix that lies the other way) by 128 bytes of the contraction.
//   rows by contraction: a load of the workgroup fills 32 rows, lane l of wavefront w the 16-byte piece l % 8 of row 8 w + l / 8; piece c of a row sits at c ^ (row / 2
//   mod 8), which spreads the 16 rows of a fragment over all LDS banks
//   KM, the other way: BK rows of ROWS columns; piece c of row k sits at c ^ key(k), so that what half a wavefront reads of 8 rows (bf16, transposing reads) or of 2 (float32) lies on all banks.
template <typename T, int ROWS, bool KM>
struct Side {
  static constexpr int ES = sizeof(T), BK = 128 / ES, LOADS = ROWS / 32, PIECES = ROWS * ES / 16;     // loads of a k-tile; KM: pieces of a row
  __amdgpu_buffer_rsrc_t rsrc;
  uint32_t voff[LOADS];
  uint32_t step;            // bytes from a k-tile to the next
  int k[LOADS], K;          // KM: rows of the loads in a k-tile, the contraction's length; otherwise k[0]: first byte of the piece, K: bytes
  static __device__ __forceinline__ int key(int k) {
    if constexpr (ES == 4) return PIECES == 32 ? 0 : PIECES == 16 ? (k & 4) << 1 : k & 4;
    else if constexpr (PIECES >= 16) return ((k & 3) | ((k >> 1) & 4)) << 1;
    else if constexpr (PIECES == 8) return (((k >> 1) & 1) | ((k >> 2) & 2)) << 1;
    else return (k >> 2) & 2;
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
  // 32 bytes of the contraction for each of the wavefront's 16 N rows (columns) from r0 on, those that the other operand's fragments take.  Fragment i's row is r0 + 16 i + lane % 16,
  // but of float32 that lies the other way r0 + N (lane % 16) + i: one read then brings N columns of a step of the contraction.
  template <int N>
  __device__ __forceinline__ void fragments(const unsigned char* st, int r0, int lane, Fragment<T> (&f)[N]) const {
    const int lgrp = lane >> 4, lrow = lane & 15;
    if constexpr (!KM) {
      const unsigned char* const row = st + (r0 + lrow) * 128;
      const int x0 = (lgrp ^ ((lane >> 1) & 7)) << 4;
#pragma unroll
      for (int i = 0; i < N; ++i) f[i].set(*(const u32x4*)(row + i * 2048 + x0), *(const u32x4*)(row + i * 2048 + (x0 ^ 64)));
    } else if constexpr (ES == 2) {
      typedef __attribute__((ext_vector_type(4))) short i16x4;
      typedef __attribute__((address_space(3))) i16x4* lds_i16x4;
      const int row = lgrp * 8 + (lrow >> 2);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int c = ((r0 + 16 * i) >> 3) + ((lrow & 3) >> 1);
        const unsigned char* const at = st + row * (ROWS * 2) + ((c ^ key(row)) << 4) + (lrow & 1) * 8;
        u32x2 v[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) v[h] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(at + ((h >> 1) * 32 + (h & 1) * 4) * (ROWS * 2))));
        f[i].set(u32x4{v[0][0], v[0][1], v[1][0], v[1][1]}, u32x4{v[2][0], v[2][1], v[3][0], v[3][1]});
      }
    } else {
      const int c = r0 + N * lrow;
      uint32_t v[8][N];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int row = (e >> 2) * 16 + lgrp * 4 + (e & 3);
        const unsigned char* const at = st + row * (ROWS * 4) + (((c >> 2) ^ key(row)) << 4) + (c & 3) * 4;
        if constexpr (N == 4) {
          const u32x4 w = *(const u32x4*)at;
#pragma unroll
          for (int i = 0; i < 4; ++i) v[e][i] = w[i];
        } else if constexpr (N == 2) {
          const u32x2 w = *(const u32x2*)at;
          v[e][0] = w[0];
          v[e][1] = w[1];
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i) v[e][i] = ((const uint32_t*)at)[i];
        }
      }
#pragma unroll
      for (int i = 0; i < N; ++i) f[i].set(u32x4{v[0][i], v[1][i], v[2][i], v[3][i]}, u32x4{v[4][i], v[5][i], v[6][i], v[7][i]});
    }
  }
};

// BM x BN tile, 4 wavefronts in a 2 x 2 grid, NS LDS stages of a k-tile of 128 bytes each, one barrier a k-tile.  NG such groups of wavefronts take a part of the
// contraction each (kper k-tiles) and are added up in order at the end.  part: of the contraction, of a whole workgroup.
// Bound by LDS and conversions between barriers: float32 (six products) 333 x 5001 x 777 34 to 37 us each (70 to 75 TFLOP/s, 420 to 450 of products), 4096 x 4096 x 4096 all three 171 to 177;
// where W is read once and little else happens, by memory: logits of 1 x 131072 x 4096 bf16 170 us, 6.3 TB/s.
template <typename T, int KIND, int BM, int BN, int NS, int NG>
__device__ __forceinline__ void class_tile(const ClassProduct& g, int kper, int pid, int part, unsigned char* all_smem) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int BK = 128 / (int)sizeof(T), A_BYTES = BM * 128, STAGE = (BM + BN) * 128, NLD = (BM + BN) / 32, MI = BM / 32, NI = BN / 32;
  constexpr bool KMA = KIND == PRODUCT_DW, KMB = KIND == PRODUCT_DX || KMA;
  const int group = NG > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) : 0;
  unsigned char* const smem = all_smem + group * (NS * STAGE);
  int tm, tn;
  tile_of(pid, (g.M + BM - 1) / BM, (g.N + BN - 1) / BN, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int t = threadIdx.x & 255, lane = t & 63, w = t >> 6, wm = w & 1, wn = w >> 1;
  const int nk = (g.K + BK - 1) / BK, k0 = (part * NG + group) * kper, k1 = k0 + kper < nk ? k0 + kper : nk;
  Side<T, BM, KMA> A;
  Side<T, BN, KMB> B;
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
  for (int kt = k0; kt < (NG > 1 ? k0 + kper : k1); ++kt) {
    // this wavefront's part of k-tile kt has landed and its reads of the last one are done; behind the barrier, everybody's
    __builtin_amdgcn_s_waitcnt(SLP_VMCNT_LGKM0((NS - 2) * NLD));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    load(kt + NS - 1, (kt - k0 + NS - 1) % NS);
    if (NG > 1 && kt >= k1) continue;            // (a shorter part takes the others' barriers)
    const unsigned char* const st = smem + (kt - k0) % NS * STAGE;
    Fragment<T> a[MI], b[NI];
    B.fragments(st + A_BYTES, wn * (BN / 2), lane, b);
    A.fragments(st, wm * (BM / 2), lane, a);
    mma<T, MI, NI>(acc, a, b);
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
    if (group == 0) {
#pragma unroll
      for (int v = 0; v < NG - 1; ++v)
#pragma unroll
        for (int i = 0; i < MI * NI; ++i) acc[i / NI][i % NI] += sums[(v * MI * NI + i) * 256];
    }
  }
  __syncthreads();                               // nobody reads LDS any more
  if (NG > 1 && group > 0) return;
  if constexpr (sizeof(T) == 4 && KMB) {
    // the columns that a lane holds lie side by side: 4 NI of them, element e of fragment j the (NI e + j)-th
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      f32x4 v[NI];
#pragma unroll
      for (int q = 0; q < NI; ++q)
#pragma unroll
        for (int r = 0; r < 4; ++r) v[q][r] = acc[i][(4 * q + r) % NI][(4 * q + r) / NI];
#pragma unroll
      for (int q = 0; q < NI; ++q) acc[i][q] = v[q];
    }
  }
  if constexpr (sizeof(T) == 2 && (KIND == PRODUCT_DX || KIND == PRODUCT_DW) && MI * NI >= 2) {
    if (!g.work && g.out_dtype == 1) {
      // bf16 leaves as whole row segments: each wavefront's part through LDS, rows of 2 NI pieces of 16 bytes, piece c of row r at c ^ (r mod 2 NI)
      constexpr int PIECES = 2 * NI, EACH = 64 / PIECES;
      const int lgrp = lane >> 4, lrow = lane & 15;
      const float alpha = *g.alpha;
      unsigned char* const st = smem + w * (MI * NI * 512);
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          const f32x4 v = acc[i][j] * alpha;
          const bf16x4 o = {(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
          *(u32x2*)(st + (16 * i + lrow) * (PIECES * 16) + (((2 * j + (lgrp >> 1)) ^ (lrow & (PIECES - 1))) << 4) + (lgrp & 1) * 8) = __builtin_bit_cast(u32x2, o);
        }
      const int c = lane % PIECES, n = n0 + wn * (BN / 2) + 8 * c;
#pragma unroll
      for (int q = 0; q < MI * NI / 2; ++q) {
        const int r = q * EACH + lane / PIECES, m = m0 + wm * (BM / 2) + r;
        const bf16x8 o = *(const bf16x8*)(st + r * (PIECES * 16) + ((c ^ (r & (PIECES - 1))) << 4));
        if (m < g.M && n < g.N) {
          bf16* const to = (bf16*)g.out + (int64_t)m * g.ldo + n;
          if (n + 8 <= g.N) ((AnyBf16x8*)to)->v = o;
          else
            for (int e = 0; e < g.N - n; ++e) to[e] = o[e];
        }
      }
      return;
    }
  }
  if constexpr (KIND >= PRODUCT_DX) {
    if (g.work || g.out_dtype == 0) {
      // float32 the same, rows of 4 NI pieces: lanes hold 4 consecutive columns, which would leave 16 bytes at a time (dW of 21 x 81199 x 2048 468 us, in whole segments 167)
      constexpr int PIECES = 4 * NI, EACH = 64 / PIECES;
      constexpr bool AROUND = sizeof(T) == 4 && KMA, BROUND = sizeof(T) == 4 && KMB;
      static_assert(MI * NI * 4096 <= NS * STAGE, "room for the wavefronts' parts");
      auto key = [](int r) { return (AROUND ? r / MI : r) & (PIECES - 1); };
      const int lgrp = lane >> 4, lrow = lane & 15;
      const float alpha = g.work ? 1.0f : *g.alpha;
      unsigned char* const st = smem + w * (MI * NI * 1024);
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          const int r = AROUND ? MI * lrow + i : 16 * i + lrow, c = BROUND ? NI * lgrp + j : 4 * j + lgrp;
          *(f32x4*)(st + r * (PIECES * 16) + ((c ^ key(r)) << 4)) = acc[i][j] * alpha;
        }
      const int64_t ld = g.work ? (g.N + 3) & ~3 : g.ldo;
      float* const out = g.work ? g.work + (int64_t)part * g.M * ld : (float*)g.out;
      const int c = lane % PIECES, n = n0 + wn * (BN / 2) + 4 * c, left = g.work ? 4 : g.N - n;
#pragma unroll
      for (int q = 0; q < MI * NI; ++q) {
        const int r = q * EACH + lane / PIECES, m = m0 + wm * (BM / 2) + r;
        f32x4 v = *(const f32x4*)(st + r * (PIECES * 16) + ((c ^ key(r)) << 4));
        if (m < g.M && n < g.N) {
          float* const to = out + (int64_t)m * ld + n;
          if (g.work && g.add) v += *(const f32x4*)to;
          store4(to, left, v);
        }
      }
      return;
    }
  }
  finish<T, KIND, MI, NI>(g, acc, m0 + wm * (BM / 2), n0 + wn * (BN / 2), lane);
#endif
}
template <typename T, int KIND, int BM, int BN, int NS, int NG>
__global__ __launch_bounds__(256 * NG) void class_tile_kernel(const ClassProduct g, int kper) {
  extern __shared__ __attribute__((aligned(16))) unsigned char all_smem[];
  class_tile<T, KIND, BM, BN, NS, NG>(g, kper, blockIdx.x, blockIdx.y, all_smem);
}
// Both gradients of P in one launch, where each takes a few small tiles: `xtiles` times x.parts workgroups on dX, the others on dW.  Neither fills the chip, and a launch behind another
// takes 3.5 us: 64 x 1000 x 512 float32 27.3 us a call in two launches, 23.6 in one.
template <typename T, int NX, int NW>
__global__ __launch_bounds__(256) void class_pair_kernel(const ClassProduct x, int xper, int xtiles, int xblocks, const ClassProduct w, int wper, int wtiles) {
  extern __shared__ __attribute__((aligned(16))) unsigned char all_smem[];
  const int at = blockIdx.x;
  if (at < xblocks) class_tile<T, PRODUCT_DX, 32, NX, 3, 1>(x, xper, at % xtiles, at / xtiles, all_smem);
  else class_tile<T, PRODUCT_DW, 32, NW, 3, 1>(w, wper, (at - xblocks) % wtiles, (at - xblocks) / wtiles, all_smem);
}

// Large bf16 products (long_tile.h).  What the epilogues of the tiles above do, with the accumulators taken out of the AGPRs a block at a time; bf16 outputs leave as whole
// row segments, staged by each wavefront in a 32 KB of the stages that is its own, rows of 256 bytes whose 16-byte piece c sits at c ^ (row mod 16).
// Bound by the matrix unit: 8192 x 131072 x 4096 logits 6.2 to 6.3 ms (1.40-1.42 PFLOP/s), dX and dW in 8 pieces 6.2 and 5.9 to 6.0 (1.42, 1.49), probabilities
// 1.43, where the vendor's product of 8192 x 16384 x 16384 reaches 1.41 to 1.55 on the same machines.  Shorter contractions pay for their epilogues, which nothing else hides: 2048 x 32000 x 4096
// logits with 262 MB of them kept 1.17, dW of 2048 rows 1.12.
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
    constexpr bool KMA = KIND == PRODUCT_DW, KMB = KIND == PRODUCT_DX || KMA;
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
        bias[j][e] = g.bias && n < g.N ? g.bias[n] : 0.0f;
      }
    const int span = colW / 128;
    const bool edge = colW + 128 > g.N;            // (uniform over the wavefront)
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
          if (edge && colW + 16 * j + 4 * lgrp + e >= g.N) z[j][e] = -INFINITY;
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
      for (int e = 0; e < 4; ++e) bias[e] = g.bias && n + e < g.N ? g.bias[n + e] : 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        asm volatile("" : "+a"(acc[i][j]));
        f32x4 p;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float z = (acc[i][j][e] + bias[e]) * g.per_t;
          p[e] = probability(z, norm[i], n + e == label[i]);
          if (norm[i].x == INFINITY || n + e >= g.N) p[e] = 0.0f;       // (also where the row holds NaN)
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

enum Tile { kLong, k128, k128x64, k64, k64by2, k32x64, k32x64by2, k32, k32by4 };
// parts: of the contraction, which share the chip.
// 256x256 tiles where they keep half of the compute units busy, long contractions sooner, of which more than 512 of 128x128 (two a compute unit) take two rounds: dW of 8192 x 9300 x 1024
// (148 tiles) 192 us / 355 on 128x128, of 8192 x 2500 x 4096 (160) 205 / 333, of 1000 x 9000 x 1024 (144) 33 / 46, logits of it 39 / 41; short ones, logits of 1000 x 9000 x 256 (144)
// 25.6 / 21.0, of 4096 x 2600 x 512 (176) 30 / 28.
// They have one workgroup a compute unit, which waits for its own stores and loads.  Where those are all there is, two or more of 128 or 64 rows do better:
//   short contractions with a large output (dW of few rows), on 256x256 / 128x128: 16 x 131072 x 4096 411 / 323 us, 64 x 32768 x 4096 109 / 80, 128 x 65536 x 2048
//   127 / 109; 256 x 32768 x 4096 161 / 172, 512 218 / 281;
//   few rows (logits), on 256x256 / 128x128 / 64x64: 1 x 131072 x 4096 216 / 180 / 170, 64 x 131072 x 1024 62 / 47 / 42, 128 x 131072 x 4096 249 / 200 / 320, 256 x
//   131072 x 1024 71 / 93 / 128; few classes (dW): 8192 x 47 x 4096 24 / 19 / 16, 128 32 / 24 / 27;
//   few rows of dX, whose W is read across: 1 x 131072 x 4096 225 / 238 / 184, 16 229 / 239 / 204, 64 252 / 270 / 255, 128 275 / 286 / 391; 64 x 131072 x 1024 62 / 62 /
//   75, 128 x 65536 x 2048 73 / 66 / 102, 128 x 32768 x 2048 46 / 36 / 42;
//   float32, which multiplies six times, on 64x64 / 32x64: logits of 8 x 131072 x 3180 572 / 430, of 21 x 81199 x 2048 290 / 261, dX of
//   8 x 131072 x 2048 368 / 274; of 21 x 81199 x 2048 on 128x128 / 32x64 290 / 175.
Tile shape_of(int kind, int dtype, int M, int N, int K, int parts = 1) {
  const int64_t nk = ((int64_t)K * (dtype == 1 ? 2 : 4) + 127) / 128 / parts;
  const int64_t t256 = tiles_of(M, N, 256, 256) * parts, t128 = tiles_of(M, N, 128, 128) * parts, t64 = tiles_of(M, N, 64, 64) * parts;
  const bool few = M <= (kind != PRODUCT_DX ? 64 : dtype == 1 ? 16 : 32);
  if (dtype == 1 && t256 >= (nk >= 16 ? 130 : 200) && nk > 2 && !few && (M > 128 || M <= 64)) return kLong;
  if (few && t64 >= 512) return dtype == 0 && M <= 32 ? k32x64 : k64;
  if (t128 >= 384) return k128;
  if (tiles_of(M, N, 128, 64) * parts >= 480) return k128x64;
  if (tiles_of(M, N, 32, 32) * parts <= 256) return nk >= 11 ? k32by4 : k32;
  if (tiles_of(M, N, 32, 64) * parts <= 256) return nk >= 7 ? k32x64by2 : k32x64;
  if (nk >= 7 && t64 <= (nk >= 32 ? 512 : nk >= 16 ? 384 : 256)) return k64by2;
  return k64;
}
// Rows and columns of a wavefront's part of a tile.
int span_rows(Tile s) { return s == kLong ? 128 : s <= k128x64 ? 64 : s <= k64by2 ? 32 : 16; }
int span_columns(Tile s) { return s == kLong ? 128 : s == k128 ? 64 : s <= k32x64by2 ? 32 : 16; }

template <typename T, int KIND, int BM, int BN, int NS, int NG>
hipError_t launch_tile(const ClassProduct& g, hipStream_t s) {
  constexpr int smem = NG * NS * (BM + BN) * 128;
  static_assert(smem >= (NG - 1) * BM * BN * 4, "room for the groups' sums");
  static std::atomic<uint64_t> done{0};
  hipError_t e = allow_lds((const void*)class_tile_kernel<T, KIND, BM, BN, NS, NG>, smem, done);
  if (e != hipSuccess) return e;
  constexpr int BK = 128 / (int)sizeof(T);
  const int nk = (g.K + BK - 1) / BK, parts = g.work ? g.parts : 1, kper = (nk + parts * NG - 1) / (parts * NG);
  hipLaunchKernelGGL((class_tile_kernel<T, KIND, BM, BN, NS, NG>), dim3((unsigned)tiles_of(g.M, g.N, BM, BN), parts), dim3(256 * NG), smem, s, g, kper);
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
template <typename T, int NX, int NW>
hipError_t launch_pair(const ClassProduct& x, const ClassProduct& w, hipStream_t s) {
  constexpr int smem = 3 * (32 + (NX > NW ? NX : NW)) * 128, BK = 128 / (int)sizeof(T);
  auto per = [](const ClassProduct& g) { const int nk = (g.K + BK - 1) / BK, parts = g.work ? g.parts : 1; return (nk + parts - 1) / parts; };
  const int xtiles = (int)tiles_of(x.M, x.N, 32, NX), wtiles = (int)tiles_of(w.M, w.N, 32, NW), xblocks = xtiles * (x.work ? x.parts : 1), wblocks = wtiles * (w.work ? w.parts : 1);
  class_pair_kernel<T, NX, NW><<<xblocks + wblocks, 256, smem, s>>>(x, per(x), xtiles, xblocks, w, per(w), wtiles);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_pair(bool x64, bool w64, const ClassProduct& x, const ClassProduct& w, hipStream_t s) {
  if (x64) return w64 ? launch_pair<T, 64, 64>(x, w, s) : launch_pair<T, 64, 32>(x, w, s);
  return w64 ? launch_pair<T, 32, 64>(x, w, s) : launch_pair<T, 32, 32>(x, w, s);
}
template <typename T, int KIND>
hipError_t launch_kind(int dtype, const ClassProduct& g, hipStream_t s) {
  switch (shape_of(KIND, dtype, g.M, g.N, g.K, g.work ? g.parts : 1)) {
    case kLong:
      if constexpr (sizeof(T) == 2) return launch_long<KIND>(g, s);
    case k128: return launch_tile<T, KIND, 128, 128, 2, 1>(g, s);
    case k128x64: return launch_tile<T, KIND, 128, 64, 2, 1>(g, s);
    case k64: return launch_tile<T, KIND, 64, 64, 2, 1>(g, s);
    case k64by2: return tiles_of(g.M, g.N, 64, 64) * (g.work ? g.parts : 1) <= 256 ? launch_tile<T, KIND, 64, 64, 3, 2>(g, s) : launch_tile<T, KIND, 64, 64, 2, 2>(g, s);
    case k32x64: return launch_tile<T, KIND, 32, 64, 3, 1>(g, s);
    case k32x64by2: return launch_tile<T, KIND, 32, 64, 3, 2>(g, s);
    case k32: return launch_tile<T, KIND, 32, 32, 4, 1>(g, s);
    default: return launch_tile<T, KIND, 32, 32, 3, 4>(g, s);
  }
}
template <typename T>
hipError_t launch_type(int dtype, int kind, const ClassProduct& g, hipStream_t s) {
  switch (kind) {
    case PRODUCT_STATS: return launch_kind<T, PRODUCT_STATS>(dtype, g, s);
    case PRODUCT_PROB: return launch_kind<T, PRODUCT_PROB>(dtype, g, s);
    case PRODUCT_Z: return launch_kind<T, PRODUCT_Z>(dtype, g, s);
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

// Parts of a contraction whose few tiles would leave most of the chip waiting for a long one, where the partial sums are few: 2 x 64 x 4096 float32 35 us in one, 6 in 16.
int z_parts(int dtype, int M, int N, int K) {
  const int nk = (K + (dtype == 1 ? 63 : 31)) / (dtype == 1 ? 64 : 32);
  if (nk < 32 || tiles_of(M, N, 128, 128) >= 200) return 0;
  int parts = class_parts(dtype, M, N, K);
  if (parts > nk / 8) parts = nk / 8;
  return parts < 2 || (int64_t)M * N * parts > 1 << 23 ? 0 : parts;
}

// Tiles of 256x256 go round by round of 256; few of them behind a few whole rounds keep most of the chip waiting, and go on smaller tiles in a launch of their own.  In one / two: logits of
// 1000 x 50001 x 1500 (784 tiles) 227 / 205 us, 2048 x 17000 x 4096 (536) 321 / 283, 4096 x 4300 x 4096 (272) 188 / 145, dW of it 183 / 156; with more rounds or more tiles left they run into each
// other anyway: dW of 2048 x 17000 x 4096 (1072) 294 / 298, 18300 (1152) 306 / 325.
int whole_rounds(int dtype, int kind, int classes, int others, int K) {
  const int M = kind == PRODUCT_DW ? classes : others, N = kind == PRODUCT_DW ? others : classes;
  const int64_t tiles = tiles_of(M, N, 256, 256), rounds = tiles / 256, across = (others + 255) / 256;
  if (shape_of(kind, dtype, M, N, K) != kLong || rounds < 1 || rounds > 3 || tiles % 256 == 0 || tiles % 256 > 64 || across > 64) return classes;
  return (int)(rounds * 256 / across) * 256;
}
int stats_spans(int dtype, int M, int N, int K) {
  const int w = span_columns(shape_of(PRODUCT_STATS, dtype, M, N, K));
  return (N + 2 * w - 1) / (2 * w) * 2;
}
int sum_parts(int dtype, int M, int N, int K) {
  const int w = span_rows(shape_of(PRODUCT_PROB, dtype, M, N, K));
  return (M + 2 * w - 1) / (2 * w) * 2;
}

static bool addressable(int dtype, int kind, const ClassProduct& g) {
  const int64_t es = dtype == 1 ? 2 : 4;
  // a tile's rows, or an operand that lies the other way, are addressed with 32-bit offsets
  const int64_t rows_a = kind == PRODUCT_DW ? g.K : 256, rows_b = kind == PRODUCT_DX || kind == PRODUCT_DW ? g.K : 256;
  if (g.M <= 0 || g.N <= 0 || g.K <= 0 || rows_a * g.lda * es >= 0x7FFFFF00 || rows_b * g.ldb * es >= 0x7FFFFF00) return false;
  return !((((uintptr_t)g.a | (uintptr_t)g.b) & 15) || g.lda * es % 16 || g.ldb * es % 16);
}
hipError_t launch_class_product(int dtype, int kind, const ClassProduct& g, hipStream_t s) {
  if (!addressable(dtype, kind, g)) return hipErrorInvalidValue;
  return dtype == 1 ? launch_type<bf16>(dtype, kind, g, s) : launch_type<float>(dtype, kind, g, s);
}
hipError_t launch_class_gradients(int dtype, const ClassProduct& x, const ClassProduct& w, bool& together, hipStream_t s) {
  auto shape = [&](int kind, const ClassProduct& g) { return shape_of(kind, dtype, g.M, g.N, g.K, g.work ? g.parts : 1); };
  const Tile sx = shape(PRODUCT_DX, x), sw = shape(PRODUCT_DW, w);
  together = (sx == k32 || sx == k32x64) && (sw == k32 || sw == k32x64);
  if (!together) return launch_class_product(dtype, PRODUCT_DX, x, s);
  if (!addressable(dtype, PRODUCT_DX, x) || !addressable(dtype, PRODUCT_DW, w)) return hipErrorInvalidValue;
  return dtype == 1 ? launch_pair<bf16>(sx == k32x64, sw == k32x64, x, w, s) : launch_pair<float>(sx == k32x64, sw == k32x64, x, w, s);
}

}  // namespace slp
