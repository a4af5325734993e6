// Which kernel a product of 8-bit matrices runs on (product.hip: e4m3 values, integers.hip: integers).
#pragma once

#include <stdint.h>

namespace slp {
namespace {

inline int64_t tiles_of(int M, int N, int BM, int BN) { return (int64_t)((M + BM - 1) / BM) * ((N + BN - 1) / BN); }

// Which kernel a product runs on.
enum Shape { kRows, kBig, k128, k128x64, k64, k64by2, k32x64, k32x64by2, k32, k32by4, kSplit, kSplit32by4 };

// Whether it is a kernel for few rows (product_rows_kernel).  Its workgroups read A as often as there are 16 rows of B, and a compute unit reads 16 rows in 0.7 us per
// 1024 k (1.2 with 16 rows of A).  Microseconds, this / tiles: 1 x 1000 x 784 2.9 / 3.9, 1 x 4096 x 8192 8.2 / 10.9, 4 x 512 x 8192 8.0 / 7.7, 1 x 1000 x
// 16384 12.3 / 8.7, 12 x 4096 x 4096 6.6 / 6.5, 8 x 2048 x 8192 9.6 / 8.1, 16 x 1000 x 2000 4.5 / 4.9, 16 x 1000 x 4000 6.9 / 6.4, 32 x 4096 x 1024 4.1 / 4.3,
// 32 x 1000 x 2000 5.7 / 5.0; with 4 fragments of A 40 x 1000 x 784 4.5 / 4.1, 64 x 64 x 256 3.6 / 3.0, 64 x 1000 x 784 4.8 / 4.1;
// many columns 16 x 16384 x 1024 6.4 / 5.5, 32 x 16384 x 512 5.6 / 4.7.
inline bool few_rows(int M, int N, int K) {
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
inline Shape shape_of(int M, int N, int K, int form, bool aligned) {
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
inline int parts_of(Shape shape, int M, int N, int K) {
  const int nk = (K + 127) / 128;
  const int64_t t = shape == kSplit ? 512 / tiles_of(M, N, 64, 64) : 256 / tiles_of(M, N, 32, 32);
  const int most = shape == kSplit ? nk / 8 : nk / 16;
  return t < most ? (int)t : most;
}

}  // namespace
}  // namespace slp
