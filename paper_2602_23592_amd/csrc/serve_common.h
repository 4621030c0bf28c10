// Shared by the entry points of include/keep_serve.h: errors, argument checks, cache formats.
#pragma once
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include "keep_internal.h"
#include "keep_serve.h"

namespace keep {

void set_init_error(const char* text);  // api.hip: message behind keep_last_error(NULL)

__attribute__((format(printf, 2, 3))) inline keep_status serve_fail(keep_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  set_init_error(buf);
  return st;
}

inline keep_status launched(const char* who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? KEEP_OK : serve_fail(KEEP_ERR_HIP, "%s: %s", who, hipGetErrorString(e));
}

inline bool is_dtype(int32_t t) { return t == KEEP_F32 || t == KEEP_BF16; }
inline int dtype_size(int32_t t) { return t == KEEP_F32 ? 4 : 2; }
inline int format_size(int32_t f) { return f == KEEP_CACHE_F32 ? 4 : f == KEEP_CACHE_BF16 ? 2 : 1; }
inline bool format_scaled(int32_t f) { return f == KEEP_CACHE_FP8 || f == KEEP_CACHE_INT8; }

// n_rows rows of `width` elements, `stride` elements apart
struct Rows {
  const void* at;
  int64_t stride, width;
};

// Whether two sets of rows share an element.  With equal strides both repeat at the stride's distance, and slices of the same wide
// rows lie beside each other though the first and last address of one enclose the other; with unequal ones that counts as
// overlapping.
inline bool overlaps(const Rows& a, const Rows& b, int64_t n_rows, int size) {
  if (n_rows < 1 || a.width < 1 || b.width < 1) return false;
  const uint64_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
  const auto span = [&](const Rows& r) { return ((uint64_t)(n_rows - 1) * (uint64_t)r.stride + (uint64_t)r.width) * (uint64_t)size; };
  if (x >= y + span(b) || y >= x + span(a)) return false;
  if (n_rows == 1 || a.stride != b.stride) return true;
  const uint64_t step = (uint64_t)a.stride * (uint64_t)size;
  const uint64_t off = y >= x ? (y - x) % step : step - 1 - (x - y - 1) % step;  // of b's rows behind a's
  return off < (uint64_t)a.width * size || off + (uint64_t)b.width * size > step;
}

// paged_cache.hip: KEEP_OK, or the status with its text set
keep_status check_cache(const keep_paged_cache* c, const char* who);

// Division of 31-bit numbers by a divisor fixed per launch: n / d = n * mul >> shift.  With l = ceil(log2 d) and
// mul = floor(2^(31 + l) / d) + 1, mul * d exceeds 2^(31 + l) by at most d <= 2^l, so the quotient is exact for n < 2^31, and
// mul < 2^33 leaves n * mul below 2^64.
struct FastDiv {
  uint64_t mul;
  uint32_t shift, d;
};
inline FastDiv fast_div(uint32_t d) {
  uint32_t l = 0;
  while ((1ull << l) < d) ++l;
  return FastDiv{(1ull << (31 + l)) / d + 1, 31 + l, d};
}
__host__ __device__ __forceinline__ uint32_t div_by(uint32_t n, FastDiv f) { return (uint32_t)((uint64_t)n * f.mul >> f.shift); }

}  // namespace keep
