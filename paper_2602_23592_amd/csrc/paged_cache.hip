// Keys and values into the pages of a cache, and back: as they are, or with 8-bit codes and one scale per token and head.
//
//   scale = max(amax * (1 / Q), 2^-126),  code = round(x / scale),  a code stands for code * scale
//
// Both directions move every value once (HBM bound).  A group of lanes owns the values of one token and head, eight each, so
// the largest magnitude is a butterfly inside the group, on the values' bit patterns: as unsigned numbers finite magnitudes <
// infinity < NaN, and a head that is not finite shows in the same reduction.  Keys and values of the same token and head are
// two independent streams of one thread.
// 33 024 tokens with 8 heads of 128, bf16 rows and int8 pages (203 MB each way): write 52 us (3.9 TB/s), read 33 (6.1 TB/s), together
// the rate of a large copy.  With a division per value the write took 61; neighbouring tokens on one XCD 56, rows requested
// before their slot is known 55.
#include <algorithm>

#include "serve_common.h"

namespace keep {

keep_status check_cache(const keep_paged_cache* c, const char* who) {
  if (!c) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: cache is NULL", who);
  if (c->format < KEEP_CACHE_F32 || c->format > KEEP_CACHE_INT8)
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: unknown cache format %d", who, c->format);
  if (c->n_pages < 1 || c->page_size < 1 || c->n_kv_heads < 1)
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: n_pages, page_size and n_kv_heads must be at least 1", who);
  if (c->head_dim < 16 || c->head_dim % 16 || c->head_dim > 256)
    return serve_fail(KEEP_ERR_SHAPE, "%s: head_dim %d is not a multiple of 16 up to 256", who, c->head_dim);
  if (c->n_kv_heads > 4096) return serve_fail(KEEP_ERR_SHAPE, "%s: more than 4096 heads", who);
  if ((int64_t)c->n_pages * c->page_size > INT32_MAX)
    return serve_fail(KEEP_ERR_SHAPE, "%s: n_pages * page_size is above 2^31 - 1 slots", who);
  const int step = 16 / format_size(c->format);
  for (const int64_t s : {c->page_stride, c->head_stride, c->token_stride})
    if (s < 0 || s % step || s > (int64_t)1 << 44)
      return serve_fail(KEEP_ERR_INVALID_ARG, "%s: a cache stride is negative or no multiple of 16 bytes", who);
  // tokens and heads must not share values; which of them lies outermost is free
  const int64_t T = c->page_size, H = c->n_kv_heads, W = c->head_dim;
  const bool tokens_inside = (T == 1 || c->token_stride >= W) && (H == 1 || c->head_stride >= (T - 1) * c->token_stride + W);
  const bool heads_inside = (H == 1 || c->head_stride >= W) && (T == 1 || c->token_stride >= (H - 1) * c->head_stride + W);
  const int64_t page = (T - 1) * c->token_stride + (H - 1) * c->head_stride + W;
  if ((!tokens_inside && !heads_inside) || (c->n_pages > 1 && c->page_stride < page))
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: the cache's strides let tokens, heads or pages overlap, or a page reach past its stride", who);
  if (!c->k || !c->v) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: the cache's k / v is NULL", who);
  if (!aligned16(c->k) || !aligned16(c->v))
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: the cache's k / v is not 16-byte aligned", who);
  if (format_scaled(c->format)) {
    if (!c->k_scale || !c->v_scale) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: an 8-bit cache needs k_scale and v_scale", who);
    if (reinterpret_cast<uintptr_t>(c->k_scale) % 4 || reinterpret_cast<uintptr_t>(c->v_scale) % 4)
      return serve_fail(KEEP_ERR_INVALID_ARG, "%s: k_scale / v_scale is not aligned", who);
  }
  return KEEP_OK;
}

namespace {

struct CacheArgs {
  keep_paged_cache c;
  const void *k_in, *v_in;  // write: rows in
  void *k_out, *v_out;      // read: rows out
  int64_t row_stride;
  const int32_t* slots;
  int n_rows, n_slots;
  FastDiv by_page;
  FastDiv by_heads;
  int group;  // lanes per (token, head): the power of two that holds head_dim / 8
};

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void load8(const bf16_t* p, float (&v)[8]) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf16_bits_to_f32((uint16_t)w[i]);
    v[2 * i + 1] = bf16_bits_to_f32((uint16_t)(w[i] >> 16));
  }
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&v)[8]) {
  *reinterpret_cast<uint4*>(p) =
      make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}

// Codes of eight values that are at most Q in magnitude, the nearest even ones: v_cvt_pk_fp8_f32 rounds so, and so does adding
// 1.5 * 2^23, which leaves the integer in the sum's lowest bits.
template <int FMT>
__device__ __forceinline__ uint2 encode8(const float (&v)[8]) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (FMT == KEEP_CACHE_FP8) {
      int u = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
      w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], u, true);
    } else {
      uint32_t u[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) u[e] = __float_as_uint(v[4 * i + e] + 12582912.f);
      const uint32_t lo = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(u[3], u[2], 0x0c0c0400u);
      w[i] = lo | hi << 16;
    }
  }
  return make_uint2(w[0], w[1]);
}
template <int FMT>
__device__ __forceinline__ void decode8(uint2 u, float (&v)[8]) {
  const uint32_t w[2] = {u.x, u.y};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (FMT == KEEP_CACHE_FP8) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
      v[4 * i] = lo[0], v[4 * i + 1] = lo[1], v[4 * i + 2] = hi[0], v[4 * i + 3] = hi[1];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * i + e] = (float)(int8_t)(w[i] >> (8 * e));
    }
  }
}

// What a thread owns: eight values of one row and head, and where they lie in the pages.
struct Place {
  bool live;
  int row, head, d;
  int64_t value, scale;  // elements into k / v, into the scales
};

__device__ __forceinline__ Place place_of(const CacheArgs& a) {
  const int lane = threadIdx.x & (a.group - 1);
  const int64_t item = ((int64_t)blockIdx.x * 256 + threadIdx.x) / a.group;  // (row, head)
  Place p{};
  p.live = item < (int64_t)a.n_rows * a.c.n_kv_heads && lane * 8 < a.c.head_dim;
  if (!p.live) return p;
  p.row = (int)div_by((uint32_t)item, a.by_heads);
  p.head = (int)item - p.row * a.c.n_kv_heads;
  p.d = lane * 8;
  const int slot = a.slots[p.row];
  p.live = slot >= 0 && slot < a.n_slots;
  if (!p.live) return p;
  const int page = (int)div_by((uint32_t)slot, a.by_page), at = slot - page * a.c.page_size;
  p.value = page * a.c.page_stride + p.head * a.c.head_stride + at * a.c.token_stride + p.d;
  p.scale = ((int64_t)page * a.c.n_kv_heads + p.head) * a.c.page_size + at;
  return p;
}

template <int FMT>
__device__ __forceinline__ void put8(void* pages, float* scales, const Place& p, const float (&v)[8], int group) {
  if constexpr (FMT == KEEP_CACHE_F32) {
    if (p.live) store8(static_cast<float*>(pages) + p.value, v);
  } else if constexpr (FMT == KEEP_CACHE_BF16) {
    if (p.live) store8(static_cast<bf16_t*>(pages) + p.value, v);
  } else {
    constexpr float Q = FMT == KEEP_CACHE_FP8 ? 448.f : 127.f;
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
    for (int o = group >> 1; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    const bool finite = top < 0x7f800000u;
    const float scale = finite ? fmaxf(__uint_as_float(top) * (1.f / Q), 1.17549435e-38f) : __uint_as_float(0x7fc00000u);
    // The quotients by one reciprocal y = 1 / scale (rounded): q0 = x y is within 1.5 ulp, q1 = q0 + (x - q0 scale) y within one,
    // so that the next remainder is exact and q2 = q1 + (x - q1 scale) y is x / scale as a division rounds it (Markstein's
    // theorem), where nothing is lost to underflow: a remainder is a multiple of 2^-47 |q| scale, so from scale = 2^-64 on only
    // quotients below 2^-38 could differ, and their code is zero.
    float u[8];
    if (scale >= 5.421010862427522e-20f) {
      const float y = 1.f / scale;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float q0 = v[e] * y, q1 = __builtin_fmaf(__builtin_fmaf(-q0, scale, v[e]), y, q0);
        u[e] = __builtin_amdgcn_fmed3f(__builtin_fmaf(__builtin_fmaf(-q1, scale, v[e]), y, q1), -Q, Q);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = finite ? fminf(fmaxf(v[e] / scale, -Q), Q) : 0.f;
    }
    if (p.live) {
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(pages) + p.value) = encode8<FMT>(u);
      if (p.d == 0) scales[p.scale] = scale;
    }
  }
}

template <typename T, int FMT>
__global__ void __launch_bounds__(256) k_cache_write(CacheArgs a) {
  const Place p = place_of(a);
  float k[8] = {}, v[8] = {};
  if (p.live) {
    const int64_t in = p.row * a.row_stride + (int64_t)p.head * a.c.head_dim + p.d;
    load8(static_cast<const T*>(a.k_in) + in, k);
    load8(static_cast<const T*>(a.v_in) + in, v);
  }
  put8<FMT>(a.c.k, a.c.k_scale, p, k, a.group);  // (whole groups are live or not, but for lanes past head_dim, which hold zeros)
  put8<FMT>(a.c.v, a.c.v_scale, p, v, a.group);
}

template <int FMT>
__device__ __forceinline__ void get8(const void* pages, const float* scales, const Place& p, float (&v)[8]) {
  if constexpr (FMT == KEEP_CACHE_F32) {
    load8(static_cast<const float*>(pages) + p.value, v);
  } else if constexpr (FMT == KEEP_CACHE_BF16) {
    load8(static_cast<const bf16_t*>(pages) + p.value, v);
  } else {
    decode8<FMT>(*reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(pages) + p.value), v);
    const float s = scales[p.scale];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= s;
  }
}

template <typename T, int FMT>
__global__ void __launch_bounds__(256) k_cache_read(CacheArgs a) {
  const Place p = place_of(a);
  if (!p.live) return;
  float k[8], v[8];
  get8<FMT>(a.c.k, a.c.k_scale, p, k);
  get8<FMT>(a.c.v, a.c.v_scale, p, v);
  const int64_t out = p.row * a.row_stride + (int64_t)p.head * a.c.head_dim + p.d;
  store8(static_cast<T*>(a.k_out) + out, k);
  store8(static_cast<T*>(a.v_out) + out, v);
}

template <typename T>
void launch_cache(bool write, const CacheArgs& a, hipStream_t s) {
  using Kernel = void (*)(CacheArgs);
  static constexpr Kernel writers[4] = {k_cache_write<T, 0>, k_cache_write<T, 1>, k_cache_write<T, 2>, k_cache_write<T, 3>};
  static constexpr Kernel readers[4] = {k_cache_read<T, 0>, k_cache_read<T, 1>, k_cache_read<T, 2>, k_cache_read<T, 3>};
  const int64_t threads = (int64_t)a.n_rows * a.c.n_kv_heads * a.group;
  hipLaunchKernelGGL((write ? writers : readers)[a.c.format], dim3((uint32_t)((threads + 255) / 256)), dim3(256), 0, s, a);
}

keep_status cache_call(const char* me, bool write, const keep_paged_cache* c, int32_t dtype, const void* k, const void* v,
                       int32_t n_rows, int64_t row_stride, const int32_t* slots, void* stream) {
  const keep_status st = check_cache(c, me);
  if (st != KEEP_OK) return st;
  if (!is_dtype(dtype)) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: unknown dtype %d", me, dtype);
  if (n_rows < 0) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: n_rows is negative", me);
  const int size = dtype_size(dtype);
  const int64_t width = (int64_t)c->n_kv_heads * c->head_dim;
  if (row_stride < width || row_stride * size % 16)
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: row_stride must hold the row's %lld values and be a multiple of 16 bytes", me,
                      (long long)width);
  if (n_rows == 0) return KEEP_OK;
  if (!k || !v || !slots) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: k / v / slots is NULL", me);
  if (!aligned16(k) || !aligned16(v)) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: k / v is not 16-byte aligned", me);
  CacheArgs a{};
  a.c = *c;
  a.k_in = k, a.v_in = v;
  a.k_out = const_cast<void*>(k), a.v_out = const_cast<void*>(v);
  a.row_stride = row_stride;
  a.slots = slots;
  a.n_slots = c->n_pages * c->page_size;
  a.by_page = fast_div((uint32_t)c->page_size);
  a.by_heads = fast_div((uint32_t)c->n_kv_heads);
  a.group = 2;
  while (a.group * 8 < c->head_dim) a.group *= 2;
  // items are numbered in 31 bits: longer calls go out in pieces
  const int32_t most = (int32_t)(((int64_t)INT32_MAX - 256) / c->n_kv_heads / a.group);
  for (int32_t r = 0; r < n_rows; r += most) {
    CacheArgs part = a;
    part.n_rows = std::min(most, n_rows - r);
    part.slots = slots + r;
    const int64_t skip = (int64_t)r * row_stride * size;
    part.k_in = static_cast<const char*>(k) + skip, part.v_in = static_cast<const char*>(v) + skip;
    part.k_out = static_cast<char*>(a.k_out) + skip, part.v_out = static_cast<char*>(a.v_out) + skip;
    if (dtype == KEEP_F32)
      launch_cache<float>(write, part, static_cast<hipStream_t>(stream));
    else
      launch_cache<bf16_t>(write, part, static_cast<hipStream_t>(stream));
    if (n_rows - r <= most) break;
  }
  return launched(me);
}

}  // namespace
}  // namespace keep

using namespace keep;

extern "C" keep_status keep_cache_write(const keep_paged_cache* cache, int32_t dtype, const void* k, const void* v,
                                        int32_t n_rows, int64_t row_stride, const int32_t* slots, void* stream) {
  return cache_call("keep_cache_write", true, cache, dtype, k, v, n_rows, row_stride, slots, stream);
}

extern "C" keep_status keep_cache_read(const keep_paged_cache* cache, int32_t dtype, void* k, void* v, int32_t n_rows,
                                       int64_t row_stride, const int32_t* slots, void* stream) {
  return cache_call("keep_cache_read", false, cache, dtype, k, v, n_rows, row_stride, slots, stream);
}
