// A 256x256 tile of a large product on 4 wavefronts of 128 x 128, one on each SIMD, accumulators in 256 AGPRs (integers.hip, class_products.hip).
#pragma once

#include <type_traits>
#include <utility>

#include "eightbit_device.h"

namespace slp {
namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4;
#define SLP_VMCNT(n) ((((n) & 15) | 0x0F70 | (((n) >> 4) << 14)))
#define SLP_VMCNT_LGKM0(n) (SLP_VMCNT(n) & 0xF0FF)

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

// f(0), f(1), ... f(N - 1) with the index as a constant.
template <typename F, int... I>
__device__ __forceinline__ void static_for_impl(F f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, typename F>
__device__ __forceinline__ void static_for(F f) { static_for_impl(f, std::make_integer_sequence<int, N>{}); }

// workgroup -> 256x256 tile.  Consecutive workgroups go round the XCDs: all of them work on one 16 x 16 region of tiles at a time where
// the tiles divide into such, on contiguous runs of tile columns 8 tiles high otherwise.
__device__ __forceinline__ void big_tile(int M, int N, int& tm, int& tn) {
  constexpr int kXcds = 8;
  const int tilesM = (M + 255) / 256, tilesN = (N + 255) / 256, pid = blockIdx.x, xcd = pid % kXcds, q = pid / kXcds;
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

// Two LDS stages of 64 KB, a k-tile of 128 bytes of each row.  A k-tile is 128 matrix instructions of 16 cycles, two sub-steps whose 16 fragments are in
// registers before they start; everything else goes between them, at most two instructions at a time:
//   instruction   0 ..  30   reads of sub-step 1
//                40          barrier X: nobody reads this k-tile's stage any more
//                42 .. 132   the 16 loads of k-tile kt + 2 into that stage (the last one in the next k-tile's time)
//                79          barrier Y: k-tile kt + 1 has landed
//                80 .. 125   reads of its sub-step 0
// Matrix instructions and loads are assembly: the accumulators stay where they are, and a load's LDS address (m0) is set in front of a matrix instruction.  They
// take B before A: a lane then holds 4 consecutive columns of one row of the output.
// KMA, KMB (bf16): the operand lies the other way, a row of 256 columns for each k, and its fragments are read with transposing LDS reads (a group of 16 lanes reads
// 4 rows of 16 columns, lane l gets the 4 values of column l), twice as many of half the size.  A stage then holds 64 rows of 512 bytes whose 16-byte piece c sits at
// c ^ 2 s(row), s = row % 4 + 4 (row / 8 % 2), which spreads the 8 rows that half a wavefront reads over all banks.
// Acc: i32x4 (bytes, v_mfma_i32_16x16x64_i8) or f32x4 (bf16, v_mfma_f32_16x16x32_bf16).  a, b: the tile's first rows, ra and rb rows of them exist, lda and ldb bytes apart; K
// bytes of a row count, read up to the next multiple of 16 (KMA, KMB: a, b: the tile's first columns, ra and rb columns, rounded up to 8, of K / 2 rows; both matrices below 2 GiB).  RAGGED
// (integers): K does not divide by 16, what lies behind it is cut off.
constexpr int kLongSmem = 2 * 512 * 128;
template <typename Acc, bool RAGGED, bool KMA = false, bool KMB = false>
__device__ __forceinline__ void long_tile(Acc (&acc)[8][8], unsigned char* smem, const void* a, const void* b, int64_t lda, int64_t ldb, int ra, int rb, int K) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr uint32_t kPast = 0x80000000u;          // byte offset past the end of every tile
  constexpr int A_BYTES = 256 * 128, STAGE = 512 * 128;
  constexpr int RD1 = 0, X = 40, LD = 42, LD_STEP = 6, Y = 79, RD0 = 80;      // instruction index of what the comment above lists
  constexpr int kOwn = (128 - LD + LD_STEP - 1) / LD_STEP;                    // loads of a k-tile that do not go out in the next one's time
  constexpr int kBeforeY = (Y - LD + LD_STEP - 1) / LD_STEP;                  // loads of k-tile kt + 2 that are out at barrier Y
  static_assert(kOwn <= 16 && LD > X && LD + 15 * LD_STEP - 128 < X && RD1 + 2 * 15 < X && RD0 + 3 * 15 < 128, "order of the events of a k-tile");
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, wm = w & 1, wn = w >> 1, lgrp = lane >> 4, lrow = lane & 15;
  const int nk = (K + 127) / 128, Kr = (K + 15) & ~15;
  // a buffer resource by words: as an operand of assembly it has to be a vector
  auto rsrc = [](const void* p, int64_t bytes) {
    const uint64_t at = (uint64_t)(uintptr_t)p;
    return i32x4{(int)(uint32_t)at, (int)(uint32_t)(at >> 32), (int)bytes, 0x00020000};
  };
  const int rows = K / 2, ca = (ra + 7) / 8 * 16, cb = (rb + 7) / 8 * 16;        // of operands that lie the other way; bytes of their columns
  const i32x4 rsrcA = rsrc(a, !KMA ? (ra - 1) * lda + Kr : rows ? (rows - 1) * lda + ca : 0), rsrcB = rsrc(b, !KMB ? (rb - 1) * ldb + Kr : rows ? (rows - 1) * ldb + cb : 0);
  // load i < 8 fills rows [32 i, 32 i + 32) of A's tile, i >= 8 of B's; wavefront w rows 8w .. 8w + 7 of those
  const int prow = w * 8 + (lane >> 3), chunk = (lane & 7) ^ ((prow >> 1) & 7);
  // the other way: load i fills rows [8 i, 8 i + 8), wavefront w rows 2w and 2w + 1 of those
  const int krow = 2 * w + (lane >> 5);
  auto kchunk = [&](int i) { return ((lane & 31) ^ (((krow & 3) | ((i & 1) << 2)) << 1)) * 16; };        // (s(8 i + krow))
  uint32_t voff[16];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (KMA) voff[i] = kchunk(i) < ca ? (uint32_t)((krow + 8 * i) * lda + kchunk(i)) : kPast;
    else voff[i] = prow + 32 * i < ra ? (uint32_t)((prow + 32 * i) * lda + chunk * 16) : kPast;
    if constexpr (KMB) voff[8 + i] = kchunk(i) < cb ? (uint32_t)((krow + 8 * i) * ldb + kchunk(i)) : kPast;
    else voff[8 + i] = prow + 32 * i < rb ? (uint32_t)((prow + 32 * i) * ldb + chunk * 16) : kPast;
  }
  typedef __attribute__((address_space(3))) void* lds_ptr_t;
  const uint32_t lds_wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(uintptr_t)(lds_ptr_t)smem + w * 1024));

#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = Acc{0, 0, 0, 0};

  // Chunks (rows) past K become zero fills: one that is past it in a k-tile is past it in all that follow.
  auto clip = [&](int kt) {
    if (kt * 128 + 128 > K) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (i < 8 ? KMA : KMB) {
          if (kt * 64 + krow + 8 * (i & 7) >= rows) voff[i] = kPast;
        } else if (kt * 128 + chunk * 16 >= Kr) {
          voff[i] = kPast;
        }
      }
    }
  };
  // The k offset is a scalar; k-tiles past the end, whose offsets are out of range already, take 0, so that no sum of the two wraps.
  struct Off { uint32_t a, b; };
  const uint32_t stepA = KMA ? (uint32_t)(64 * lda) : 128u, stepB = KMB ? (uint32_t)(64 * ldb) : 128u;
  auto koff_of = [&](int kt) { const uint32_t k = (uint32_t)(kt < nk ? kt : 0); return Off{k * stepA, k * stepB}; };
  // The statements name the m0 they set, so that one set by the compiler for an access of its own does not pass for still set behind them; it
  // warns of every register it reserves.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
#define SLP_LOAD "s_add_u32 m0, %[base], %[row]\n\t"
#define SLP_LOAD_ARGS(i, base_, koff_)                                                                                             \
  [base] "s"(base_), [row] "i"((i) < 8 ? (i) * 4096 : A_BYTES + ((i) - 8) * 4096), [off] "v"(voff[i]), [rsrc] "s"((i) < 8 ? rsrcA : rsrcB), \
      [koff] "s"((i) < 8 ? (koff_).a : (koff_).b)
  auto load = [&](int i, uint32_t base, const Off& koff) {
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
  // the other way: the address of fragment f's columns is that of the first with the piece's number ^ 2 f
  typedef __attribute__((ext_vector_type(4))) short i16x4;
  typedef __attribute__((address_space(3))) i16x4* lds_i16x4;
  uint32_t ka[8], kb[8];
  {
    const uint32_t at = (uint32_t)((lgrp * 8 + (lrow >> 2)) * 512 + (lrow & 1) * 8), s = (uint32_t)((lrow >> 2) | ((lgrp & 1) << 2)), piece = (uint32_t)((lrow & 3) >> 1);
#pragma unroll
    for (int f = 0; f < 8; ++f) {
      ka[f] = at + ((((uint32_t)wm * 16 + piece) ^ ((s ^ f) << 1)) << 4);
      kb[f] = A_BYTES + at + ((((uint32_t)wn * 16 + piece) ^ ((s ^ f) << 1)) << 4);
    }
  }
  constexpr Walk walk;
  constexpr int kReads = (KMA ? 16 : 8) + (KMB ? 16 : 8);
  // read r of a sub-step's, fragments in the order of their first use
  struct Reads {
    int f[32], half[32];         // (half 2: the fragment in one)
    constexpr Reads() : f(), half() {
      const Walk order;
      int n = 0;
      for (int i = 0; i < 16; ++i) {
        const int fr = order.first[i];
        if (fr < 8 ? KMA : KMB) {
          f[n] = fr, half[n++] = 0;
          f[n] = fr, half[n++] = 1;
        } else {
          f[n] = fr, half[n++] = 2;
        }
      }
    }
  };
  constexpr Reads reads;
  auto read = [&](int stage, int kk, auto rc) {
    constexpr int f = reads.f[decltype(rc)::value], half = reads.half[decltype(rc)::value];
    if constexpr (half == 2) {
      if constexpr (f < 8) af[kk][f] = *(const u32x4*)(smem + stage * STAGE + fa[kk] + f * 2048);
      else bfr[kk][f - 8] = *(const u32x4*)(smem + stage * STAGE + fb[kk] + (f - 8) * 2048);
    } else {
      const u32x2 v = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)(smem + stage * STAGE + (f < 8 ? ka[f & 7] : kb[f & 7]) + kk * 16384 + half * 2048)));
      u32x4& to = f < 8 ? af[kk][f & 7] : bfr[kk][f & 7];
      to[2 * half] = v[0];
      to[2 * half + 1] = v[1];
    }
  };
  auto mma = [&](int kk, int ia, int ib) {
    if constexpr (std::is_same_v<Acc, i32x4>) asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(acc[ia][ib]) : "v"(bfr[kk][ib]), "v"(af[kk][ia]));
    else asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc[ia][ib]) : "v"(bfr[kk][ib]), "v"(af[kk][ia]));
  };
  auto mma_load = [&](int kk, int ia, int ib, int i, uint32_t base, const Off& koff) {        // the matrix instruction is the wait state that m0 needs
    if constexpr (std::is_same_v<Acc, i32x4>)
      asm volatile(SLP_LOAD "v_mfma_i32_16x16x64_i8 %[acc], %[b], %[a], %[acc]\n\tbuffer_load_dwordx4 %[off], %[rsrc], %[koff] offen lds"
                   : [acc] "+a"(acc[ia][ib]) : [b] "v"(bfr[kk][ib]), [a] "v"(af[kk][ia]), SLP_LOAD_ARGS(i, base, koff) : "memory", "scc", "m0");
    else
      asm volatile(SLP_LOAD "v_mfma_f32_16x16x32_bf16 %[acc], %[b], %[a], %[acc]\n\tbuffer_load_dwordx4 %[off], %[rsrc], %[koff] offen lds"
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
      if (chunk == (K >> 4 & 7)) {
        const u32x4 mask = first_bytes(K & 15);
        u32x4* const p = (u32x4*)(smem + (kt & 1) * STAGE + A_BYTES + w * 1024 + lane * 16);
#pragma unroll 4
        for (int i = 0; i < 8; ++i) p[i * 256] &= mask;
      }
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(kLgkm0);
    }
  };
  clip(0);
  static_for<16>([&](auto i) { load(i, lds_wave, Off{0u, 0u}); });
  clip(1);
  static_for<kOwn>([&](auto i) { load(i, lds_wave + STAGE, koff_of(1)); });
  cut(0, std::integral_constant<int, SLP_VMCNT(kOwn)>{});
  SLP_BARRIER(SLP_VMCNT(kOwn));
  static_for<kReads>([&](auto r) { read(0, 0, r); });
  for (int kt = 0; kt < nk; ++kt) {
    const int cur = kt & 1, nxt = cur ^ 1;
    const uint32_t base1 = lds_wave + nxt * STAGE, base2 = lds_wave + cur * STAGE;
    const Off koff1 = koff_of(kt + 1), koff2 = koff_of(kt + 2);
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
      if constexpr (kReads == 16) {
        if constexpr (p >= RD1 && (p - RD1) % 2 == 0 && (p - RD1) / 2 < 16) read(cur, 1, std::integral_constant<int, (p - RD1) / 2>{});
        if constexpr (p >= RD0 && (p - RD0) % 3 == 0 && (p - RD0) / 3 < 16) read(nxt, 0, std::integral_constant<int, (p - RD0) / 3>{});
      } else {
        // more of them, evenly over the first 34 and the last 46
        if constexpr (p < 34) static_for<(p + 1) * kReads / 34 - p * kReads / 34>([&](auto i) { read(cur, 1, std::integral_constant<int, p * kReads / 34 + decltype(i)::value>{}); });
        if constexpr (p >= RD0 && p < RD0 + 46)
          static_for<(p - RD0 + 1) * kReads / 46 - (p - RD0) * kReads / 46>([&](auto i) { read(nxt, 0, std::integral_constant<int, (p - RD0) * kReads / 46 + decltype(i)::value>{}); });
      }
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
#endif
}

}  // namespace
}  // namespace slp
