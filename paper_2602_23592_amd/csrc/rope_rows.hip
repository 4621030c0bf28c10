// Rotary positions on rows of queries and keys: half and interleaved pairs, part of a head, any table of frequencies.
//
// A pair (x1, x2) at angle a becomes (m (x1 cos a - x2 sin a), m (x2 cos a + x1 sin a)); all heads of a row share the
// row's rot_dim / 2 angles.  The kernel moves each value once in and once out (HBM bound): a workgroup first puts the cosines and
// sines of its rows into LDS (angle, reduction and both functions in double: at position 1e6 a binary32 angle is off by 0.03
// rad), then streams the rows' heads in 16-byte pieces, a thread holding both halves of its pairs.
// 33 024 rows of 40 + 8 heads of 128 in bf16 (812 MB in and out): 155 us, 5.2 TB/s, where a copy of 4 GiB moves 4.7; 8 rows: 3 us
// behind 8 us of the call itself.
#include <algorithm>

#include "serve_common.h"

namespace keep {
namespace {

template <typename T>
struct Piece;  // 16 bytes of values
template <>
struct Piece<float> {
  static constexpr int N = 4;
  __device__ static void load(const float* p, float (&v)[4]) {
    const float4 u = *reinterpret_cast<const float4*>(p);
    v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w;
  }
  __device__ static void store(float* p, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
};
template <>
struct Piece<bf16_t> {
  static constexpr int N = 8;
  __device__ static void load(const bf16_t* p, float (&v)[8]) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = bf16_bits_to_f32((uint16_t)w[i]);
      v[2 * i + 1] = bf16_bits_to_f32((uint16_t)(w[i] >> 16));
    }
  }
  __device__ static void store(bf16_t* p, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(p) =
        make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  }
};

struct RopeArgs {
  const void *q_in, *k_in;
  void *q_out, *k_out;
  int64_t q_in_stride, q_out_stride, k_in_stride, k_out_stride;
  const int32_t* positions;
  const double* freq;
  int n_rows, n_q_heads, n_heads;  // n_heads: of queries and keys together
  int head_dim, half;              // half = rot_dim / 2
  int rows_per_block;
  float magnitude;
  bool copy_rest;                  // out is another buffer: values from rot_dim on are moved too
};

// VEC: pieces of 16 bytes (addresses, strides, head_dim and the halves allow them), else single pairs.
template <typename T, bool HALF, bool VEC>
__global__ void __launch_bounds__(256) k_rope_rows(RopeArgs a) {
  extern __shared__ float2 table[];  // [rows of the workgroup][half]: cos, sin
  const int row0 = blockIdx.x * a.rows_per_block;
  const int rows = min(a.rows_per_block, a.n_rows - row0);
  for (int i = threadIdx.x; i < rows * a.half; i += 256) {
    const int r = i / a.half, j = i - r * a.half;
    const double angle = (double)a.positions[row0 + r] * a.freq[j];
    double s, c;
    sincos(angle, &s, &c);
    table[i] = make_float2((float)(c * a.magnitude), (float)(s * a.magnitude));
  }
  __syncthreads();
  constexpr int N = VEC ? Piece<T>::N : 1;
  // items of a head: pieces of N pairs (HALF: N values of either half; interleaved: N / 2 pairs), then pieces of what is left
  const int turned = VEC && !HALF ? 2 * a.half / N : (a.half + N - 1) / N;
  const int rest = a.copy_rest ? (a.head_dim - 2 * a.half) / N : 0;
  const int per_head = turned + rest, per_row = per_head * a.n_heads;
  for (int i = threadIdx.x; i < rows * per_row; i += 256) {
    const int r = i / per_row, h = (i - r * per_row) / per_head, c = i - r * per_row - h * per_head;
    const bool is_q = h < a.n_q_heads;
    const int64_t row = row0 + r, head = (int64_t)(is_q ? h : h - a.n_q_heads) * a.head_dim;
    const T* x = static_cast<const T*>(is_q ? a.q_in : a.k_in) + row * (is_q ? a.q_in_stride : a.k_in_stride) + head;
    T* y = static_cast<T*>(is_q ? a.q_out : a.k_out) + row * (is_q ? a.q_out_stride : a.k_out_stride) + head;
    const float2* cs = table + r * a.half;
    if (c >= turned) {
      const int d = 2 * a.half + (c - turned) * N;
      if constexpr (VEC)
        *reinterpret_cast<uint4*>(y + d) = *reinterpret_cast<const uint4*>(x + d);
      else
        y[d] = x[d];
    } else if constexpr (!VEC) {
      const int d1 = HALF ? c : 2 * c, d2 = HALF ? c + a.half : 2 * c + 1;
      const float x1 = ldf(x + d1), x2 = ldf(x + d2);
      stf(y + d1, x1 * cs[c].x - x2 * cs[c].y);
      stf(y + d2, x2 * cs[c].x + x1 * cs[c].y);
    } else if constexpr (HALF) {
      float x1[N], x2[N], y1[N], y2[N];
      Piece<T>::load(x + c * N, x1);
      Piece<T>::load(x + a.half + c * N, x2);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float2 t = cs[c * N + e];
        y1[e] = x1[e] * t.x - x2[e] * t.y;
        y2[e] = x2[e] * t.x + x1[e] * t.y;
      }
      Piece<T>::store(y + c * N, y1);
      Piece<T>::store(y + a.half + c * N, y2);
    } else {
      float v[N], w[N];
      Piece<T>::load(x + c * N, v);
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        const float2 t = cs[(c * N + e) >> 1];
        w[e] = v[e] * t.x - v[e + 1] * t.y;
        w[e + 1] = v[e + 1] * t.x + v[e] * t.y;
      }
      Piece<T>::store(y + c * N, w);
    }
  }
}

template <typename T>
void launch_rope_rows(RopeArgs a, bool half, bool vec, hipStream_t s) {
  const dim3 grid((a.n_rows + a.rows_per_block - 1) / a.rows_per_block);
  const size_t lds = (size_t)a.rows_per_block * a.half * sizeof(float2);
  const auto kernel = half ? (vec ? k_rope_rows<T, true, true> : k_rope_rows<T, true, false>)
                           : (vec ? k_rope_rows<T, false, true> : k_rope_rows<T, false, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(256), lds, s, a);
}

}  // namespace
}  // namespace keep

using namespace keep;

extern "C" keep_status keep_rope_frequencies(const keep_rope_desc* d, double* freq, float* magnitude) {
  const char* me = "keep_rope_frequencies";
  if (!d || !freq || !magnitude) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: desc / freq / magnitude is NULL", me);
  if (d->rot_dim < 2 || d->rot_dim % 2)
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: rot_dim %d must be even and positive", me, d->rot_dim);
  if (d->scaling < KEEP_ROPE_PLAIN || d->scaling > KEEP_ROPE_PARTS)
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: unknown scaling %d", me, d->scaling);
  if (!(d->theta > 0.0) || !isfinite(d->theta)) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: theta must be positive", me);
  if (d->scaling != KEEP_ROPE_PLAIN && (!(d->factor >= 1.0) || !isfinite(d->factor)))
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: factor must be at least 1", me);
  const bool parts = d->scaling == KEEP_ROPE_PARTS;
  if (parts && (d->trained_len < 1 || !(d->slow >= 0.0) || !(d->fast > d->slow) || !isfinite(d->fast)))
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: PARTS needs trained_len >= 1 and fast > slow >= 0", me);
  const double r = d->rot_dim;
  double theta = d->theta;
  if (d->scaling == KEEP_ROPE_BASE && d->rot_dim > 2) theta *= pow(d->factor, r / (r - 2.0));
  for (int j = 0; j < d->rot_dim / 2; ++j) {
    double f = pow(theta, -2.0 * j / r);
    if (d->scaling == KEEP_ROPE_LINEAR) f /= d->factor;
    if (parts) {
      const double turns = d->trained_len * f / (2.0 * M_PI);
      const double keep = std::min(1.0, std::max(0.0, (turns - d->slow) / (d->fast - d->slow)));
      f = (1.0 - keep) * f / d->factor + keep * f;
    }
    freq[j] = f;
  }
  *magnitude = parts ? (float)(0.1 * log(d->factor) + 1.0) : 1.f;
  return KEEP_OK;
}

extern "C" keep_status keep_rope_rows(const keep_rope_rows_desc* d, const void* q_in, void* q_out, const void* k_in,
                                      void* k_out, const int32_t* positions, const double* freq, void* stream) {
  const char* me = "keep_rope_rows";
  if (!d) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: desc is NULL", me);
  if (!is_dtype(d->dtype)) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: unknown dtype %d", me, d->dtype);
  if (d->layout != KEEP_ROPE_HALF && d->layout != KEEP_ROPE_INTERLEAVED)
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: unknown layout %d", me, d->layout);
  if (d->n_rows < 0 || d->n_q_heads < 0 || d->n_kv_heads < 0 || d->n_q_heads + (int64_t)d->n_kv_heads < 1)
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: negative n_rows or heads, or no heads at all", me);
  if (d->head_dim < 1 || d->head_dim > 1024)
    return serve_fail(KEEP_ERR_SHAPE, "%s: head_dim %d outside [1, 1024]", me, d->head_dim);
  if (d->rot_dim < 2 || d->rot_dim % 2 || d->rot_dim > d->head_dim)
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: rot_dim %d must be even, 2 .. head_dim", me, d->rot_dim);
  const int64_t qw = (int64_t)d->n_q_heads * d->head_dim, kw = (int64_t)d->n_kv_heads * d->head_dim;
  if (qw + kw > INT32_MAX / 16) return serve_fail(KEEP_ERR_SHAPE, "%s: rows of %lld values", me, (long long)(qw + kw));
  const int size = dtype_size(d->dtype);
  const struct {
    const void* in;
    void* out;
    int64_t w, is, os;
  } parts[2] = {{q_in, q_out, qw, d->q_in_stride, d->q_out_stride}, {k_in, k_out, kw, d->k_in_stride, d->k_out_stride}};
  bool vec = d->head_dim * size % 16 == 0 && (d->layout == KEEP_ROPE_HALF ? d->rot_dim / 2 : d->rot_dim) * size % 16 == 0;
  bool copy_rest = false;
  if (d->n_rows > 0 && (!positions || !freq)) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: positions / freq is NULL", me);
  for (const auto& p : parts) {
    if (!p.w) continue;
    if (p.is < p.w || p.os < p.w)
      return serve_fail(KEEP_ERR_INVALID_ARG, "%s: a row stride is shorter than the row's %lld values", me, (long long)p.w);
    if (d->n_rows == 0) continue;
    if (!p.in || !p.out) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: a pointer of queries or keys is NULL", me);
    if (reinterpret_cast<uintptr_t>(p.in) % size || reinterpret_cast<uintptr_t>(p.out) % size)
      return serve_fail(KEEP_ERR_INVALID_ARG, "%s: a pointer is not aligned to its elements", me);
    if (p.in != p.out || p.is != p.os) {
      if (overlaps({p.in, p.is, p.w}, {p.out, p.os, p.w}, d->n_rows, size))
        return serve_fail(KEEP_ERR_INVALID_ARG, "%s: input and output overlap without being the same rows", me);
      copy_rest = true;
    }
    vec = vec && aligned16(p.in) && aligned16(p.out) && p.is * size % 16 == 0 && p.os * size % 16 == 0;
  }
  if (d->n_rows == 0) return KEEP_OK;
  // queries beside keys: rows that one of them writes belong to it alone
  const Rows qi{q_in, d->q_in_stride, qw}, qo{q_out, d->q_out_stride, qw}, ki{k_in, d->k_in_stride, kw}, ko{k_out, d->k_out_stride, kw};
  if (overlaps(qo, ki, d->n_rows, size) || overlaps(qo, ko, d->n_rows, size) || overlaps(qi, ko, d->n_rows, size))
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: rows of queries and of keys overlap", me);
  RopeArgs a{q_in, k_in, q_out, k_out, d->q_in_stride, d->q_out_stride, d->k_in_stride, d->k_out_stride, positions, freq,
             d->n_rows, d->n_q_heads, d->n_q_heads + d->n_kv_heads, d->head_dim, d->rot_dim / 2, 1, d->magnitude, copy_rest};
  // one row per workgroup while rows are fewer than the chip holds workgroups, then four: the table's 64 pairs of a
  // 128-value head fill the 256 threads
  a.rows_per_block = d->n_rows >= 8192 ? 4 : 1;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (d->dtype == KEEP_F32)
    launch_rope_rows<float>(a, d->layout == KEEP_ROPE_HALF, vec, s);
  else
    launch_rope_rows<bf16_t>(a, d->layout == KEEP_ROPE_HALF, vec, s);
  return launched(me);
}
