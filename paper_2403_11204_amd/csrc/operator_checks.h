// Argument checks that the operators' host code shares (operators.hip, losses.hip).
#pragma once

#include "host_errors.h"

#include <stdint.h>

namespace slp {
namespace {

constexpr int kMaxSide = 1 << 24;
constexpr int64_t kMaxLd = (int64_t)1 << 40;

inline bool known(int dt) { return dt == SLP_F32 || dt == SLP_BF16; }
inline size_t size_of(int dt) { return dt == SLP_BF16 ? 2 : 4; }
inline bool off(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

// A float32 or bf16 matrix with rows of `cols` elements.
inline int check_dense(const char* who, const char* what, const void* p, int64_t ld, int cols, int dt) {
  if (ld < cols || ld > kMaxLd) return fail(SLP_ERR_SHAPE, "%s: leading dimension %lld of %s, rows of %d", who, (long long)ld, what, cols);
  if (off(p, size_of(dt))) return fail(SLP_ERR_ALLOC, "%s: %s is not on an element's boundary", who, what);
  return SLP_OK;
}

inline int check_work(const char* who, const void* p, size_t bytes, size_t need) {
  if (need && (!p || bytes < need || off(p, 256)))
    return fail(SLP_ERR_ALLOC, "%s: workspace of %zu bytes (256-byte aligned) needed, %zu given", who, need, p ? bytes : (size_t)0);
  return SLP_OK;
}

#define SLP_CHECK(expr)         \
  do {                          \
    const int rc__ = (expr);    \
    if (rc__) return rc__;      \
  } while (0)

}  // namespace
}  // namespace slp
