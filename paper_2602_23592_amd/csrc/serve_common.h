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

// bytes [a, a + na) and [b, b + nb) share an address
inline bool overlaps(const void* a, uint64_t na, const void* b, uint64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return na && nb && x < y + nb && y < x + na;
}

// bytes from the first row to the end of the last one
inline uint64_t row_span(int64_t n_rows, int64_t stride, int64_t width, int size) {
  return n_rows > 0 ? ((uint64_t)(n_rows - 1) * (uint64_t)stride + (uint64_t)width) * (uint64_t)size : 0;
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
