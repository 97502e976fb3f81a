// Host-side helpers for the C ABI implementation.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "fastcoder.h"

namespace fc {

// Workspace carving: hands out 256-byte aligned slices of a caller buffer.
struct Carver {
  char* base;
  size_t used;
  explicit Carver(void* p) : base((char*)p), used(0) {}
  template <typename T>
  T* take(size_t count) {
    used = (used + 255) & ~(size_t)255;
    T* r = base ? (T*)(base + used) : nullptr;
    used += count * sizeof(T);
    return r;
  }
};

// Bytes that a call reads or writes (p null: none).
struct Span {
  const void* p;
  uint64_t n;
};
// Whether nothing written shares a byte with anything else that the call is given.
template <size_t W, size_t R>
inline bool apart(const Span (&written)[W], const Span (&read)[R]) {
  const auto meet = [](const Span& a, const Span& b) {
    const uint64_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return a.p && b.p && a.n && b.n && x < y + b.n && y < x + a.n;
  };
  for (size_t i = 0; i < W; ++i) {
    for (size_t j = 0; j < R; ++j)
      if (meet(written[i], read[j])) return false;
    for (size_t j = 0; j < i; ++j)
      if (meet(written[i], written[j])) return false;
  }
  return true;
}
// Of rows that lie `stride` elements of two bytes apart.
inline Span rows_span(const void* p, int64_t rows, int64_t stride, int64_t len) {
  return Span{p, rows > 0 ? 2 * (uint64_t)((rows - 1) * stride + len) : 0};
}

inline fc_status launch_status() {
  hipError_t e = hipGetLastError();
  return e == hipSuccess ? FC_OK : FC_ERR_DEVICE;
}

}  // namespace fc

#define FC_CHECK_HIP(expr)                 \
  do {                                     \
    if ((expr) != hipSuccess) {            \
      (void)hipGetLastError();             \
      return FC_ERR_DEVICE;                \
    }                                      \
  } while (0)

#define FC_CHECK_LAUNCH()                  \
  do {                                     \
    if (hipGetLastError() != hipSuccess) { \
      return FC_ERR_DEVICE;                \
    }                                      \
  } while (0)
