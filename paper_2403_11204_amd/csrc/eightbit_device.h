// Device helpers of the 8-bit operators: vectors of 8 elements at any alignment, e4m3 values and their power-of-two scales.
#pragma once

#include "eightbit.h"

namespace slp {
namespace {

typedef __bf16 bf16;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

// Vectors that start at any element of a row (global memory takes them at any address).
struct __attribute__((packed, aligned(2))) AnyBf16x8 { bf16x8 v; };
struct __attribute__((packed, aligned(2))) AnyBf16x4 { bf16x4 v; };
struct __attribute__((packed, aligned(4))) AnyF32x4 { f32x4 v; };

// v[j] = p[j], 0 for j >= n
__device__ __forceinline__ void load8(const bf16* p, int n, float (&v)[8]) {
  if (n >= 8) {
    const bf16x8 x = ((const AnyBf16x8*)p)->v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)x[j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? (float)p[j] : 0.0f;
  }
}
__device__ __forceinline__ void load8(const float* p, int n, float (&v)[8]) {
  if (n >= 8) {
    const f32x4 a = ((const AnyF32x4*)p)->v, b = ((const AnyF32x4*)(p + 4))->v;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = a[j];
      v[4 + j] = b[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? p[j] : 0.0f;
  }
}
// p[j] = v[j] for j < n, rounded to the type
__device__ __forceinline__ void store8(bf16* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    bf16x8 x;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (bf16)v[j];
    ((AnyBf16x8*)p)->v = x;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = (bf16)v[j];
  }
}
__device__ __forceinline__ void store8(float* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    ((AnyF32x4*)p)->v = f32x4{v[0], v[1], v[2], v[3]};
    ((AnyF32x4*)(p + 4))->v = f32x4{v[4], v[5], v[6], v[7]};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = v[j];
  }
}

// 8 elements as they are in memory.
template <typename T> struct Raw;
template <> struct Raw<bf16> { bf16x8 v; };
template <> struct Raw<float> { f32x4 v[2]; };
__device__ __forceinline__ void fetch8(const bf16* p, int n, Raw<bf16>& r) {
  if (n >= 8) r.v = ((const AnyBf16x8*)p)->v;
  else {
#pragma unroll
    for (int j = 0; j < 8; ++j) r.v[j] = j < n ? p[j] : (bf16)0.0f;
  }
}
__device__ __forceinline__ void fetch8(const float* p, int n, Raw<float>& r) {
  if (n >= 8) {
    r.v[0] = ((const AnyF32x4*)p)->v;
    r.v[1] = ((const AnyF32x4*)(p + 4))->v;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) r.v[j / 4][j % 4] = j < n ? p[j] : 0.0f;
  }
}
__device__ __forceinline__ float item(const Raw<bf16>& r, int j) { return (float)r.v[j]; }
__device__ __forceinline__ float item(const Raw<float>& r, int j) { return r.v[j / 4][j % 4]; }

// Lane i of a row of 16 takes the value of the lane that the control names.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
}
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t max_of_16(uint32_t x) {
  x = umax(x, dpp<kSwap1>(x));
  x = umax(x, dpp<kSwap2>(x));
  x = umax(x, dpp<kHalfMirror>(x));
  return umax(x, dpp<kMirror>(x));
}
// Over the lanes l, l ^ 16, l ^ 32 and l ^ 48: two instructions that exchange halves and quarters of the wavefront between two registers.
__device__ __forceinline__ uint32_t max_of_rows(uint32_t x) {
  u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(x, x, false, false));
  x = umax(r[0], r[1]);
  r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(x, x, false, false));
  return umax(r[0], r[1]);
}
__device__ __forceinline__ float sum_of_rows(float x) {
  uint32_t u = __builtin_bit_cast(uint32_t, x);
  u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(u, u, false, false));
  uint32_t a = r[0], b = r[1];         // (a bit cast of a vector's element takes the first one's)
  u = __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
  r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(u, u, false, false));
  a = r[0];
  b = r[1];
  return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}
template <int CTRL>
__device__ __forceinline__ float add_dpp(float x) { return x + __builtin_bit_cast(float, dpp<CTRL>(__builtin_bit_cast(uint32_t, x))); }
__device__ __forceinline__ float sum_of_16(float x) {
  x = add_dpp<kSwap1>(x);
  x = add_dpp<kSwap2>(x);
  x = add_dpp<kHalfMirror>(x);
  return add_dpp<kMirror>(x);
}
__device__ __forceinline__ float sum_of_64(float x) { return sum_of_rows(sum_of_16(x)); }

// |v| as an integer that orders like the value, infinities and NaN above all others
__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu; }
// The scale 2^e of a block as e + 127: the least e >= -127 with max|x| <= 448 2^e (448 = 1.75 2^8, the largest e4m3 value).  With max|x| =
// f 2^k, 1 <= f < 2, e is k - 8, one more where f > 1.75: the carry of adding 0.25 - 2^-23 to the fraction.  A block that holds an infinity
// or a NaN gets 255, the scale's own NaN: everything computed from it is NaN, as it would be from the block itself.
__device__ __forceinline__ uint32_t scale_of(uint32_t amax) {
  const int e = (int)((amax + 0x1FFFFFu) >> 23) - 8;
  return amax >= 0x7F800000u ? 255u : (uint32_t)(e > 0 ? e : 0);
}
// The scale as the conversions take it, which read its exponent's bits.
__device__ __forceinline__ float scale_value(uint32_t scale) { return __builtin_bit_cast(float, scale << 23); }
// Values over their scale to e4m3, round to nearest even.  None is above 448, so nothing saturates.
typedef __attribute__((ext_vector_type(2))) short i16x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d, float scale) {
  i16x2 o = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(i16x2{0, 0}, a, b, scale, false);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(o, c, d, scale, true);
  return __builtin_bit_cast(uint32_t, o);
}
__device__ __forceinline__ uint32_t to_e4m3(uint32_t ab, uint32_t cd, float scale) {        // pairs of bf16
  i16x2 o = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(i16x2{0, 0}, __builtin_bit_cast(bf16x2, ab), scale, false);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(o, __builtin_bit_cast(bf16x2, cd), scale, true);
  return __builtin_bit_cast(uint32_t, o);
}
__device__ __forceinline__ u32x2 to_e4m3(const float (&v)[8], float scale) {
  return u32x2{to_e4m3(v[0], v[1], v[2], v[3], scale), to_e4m3(v[4], v[5], v[6], v[7], scale)};
}

}  // namespace
}  // namespace slp
