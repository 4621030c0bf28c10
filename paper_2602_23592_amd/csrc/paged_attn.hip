// Attention of new tokens over a cache in pages: the entry point, the join of cut jobs, and the kernel for every type and
// head width (fp32 matrix instruction).  paged_attn.h says how the work is dealt.
//
// One pass over the keys with a running maximum m and sum l per query row (log2 domain):
//   m' = max(m, s),  l' = l 2^(m - m') + sum 2^(s - m'),  O' = O 2^(m - m') + 2^(s - m') V,   result O / l.
#include <algorithm>
#include <type_traits>

#include "paged_attn.h"

namespace keep {
namespace {

using f32x4 = paged_f32x4;

constexpr int GT_KEYS = 64;

// Four values as they lie in memory, from element i on, and the numbers they stand for
template <int FORMAT>
__device__ __forceinline__ uint4 load_raw(const void* p, int64_t i) {
  if (FORMAT == KEEP_CACHE_F32) return *reinterpret_cast<const uint4*>(static_cast<const float*>(p) + i);
  if (FORMAT == KEEP_CACHE_BF16) {
    const uint2 u = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + i);
    return make_uint4(u.x, u.y, 0, 0);
  }
  return make_uint4(*reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(p) + i), 0, 0, 0);
}
template <int FORMAT>
__device__ __forceinline__ f32x4 value_of(uint4 u, float scale) {
  if (FORMAT == KEEP_CACHE_F32)
    return f32x4{__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w)};
  if (FORMAT == KEEP_CACHE_BF16)
    return f32x4{__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                 __uint_as_float(u.y & 0xffff0000u)};
  if (FORMAT == KEEP_CACHE_FP8) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)u.x, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)u.x, true);
    return f32x4{lo[0] * scale, lo[1] * scale, hi[0] * scale, hi[1] * scale};
  }
  return f32x4{(float)(int8_t)u.x * scale, (float)(int8_t)(u.x >> 8) * scale, (float)(int8_t)(u.x >> 16) * scale,
               (float)(int8_t)(u.x >> 24) * scale};
}

__device__ __forceinline__ bool finite4(f32x4 v) {
  bool ok = true;
#pragma unroll
  for (int e = 0; e < 4; ++e) ok = ok && (__float_as_uint(v[e]) & 0x7f800000u) != 0x7f800000u;
  return ok;
}

// A thread's share of a key tile: every fourth four values of one key
template <int ND>
struct GenericShare {
  int64_t at, scale_at;  // of the tile on its way; -1: the key lies behind the sequence's end
  int page;              // of the key in the tile after that (a tile's loads would else wait for their page's)
  uint4 raw[ND];
  float scale;
};
template <int ND>
__device__ __forceinline__ void generic_page(const PagedArgs& a, const PagedSeq& q, const int32_t* table, int kt,
                                             GenericShare<ND>& f) {
  const int key = kt * GT_KEYS + (int)(threadIdx.x >> 2);
  if (key < q.len) f.page = table[div_by(key, a.by_page)];
}
template <int ND>
__device__ __forceinline__ void generic_locate(const PagedArgs& a, const PagedPlace& p, const PagedSeq& q, const int32_t* table,
                                               int kt, GenericShare<ND>& f) {
  const int key = kt * GT_KEYS + (int)(threadIdx.x >> 2);
  f.at = -1;
  if (key >= q.len) return;
  const int page = min(max(f.page, 0), a.c.n_pages - 1), in = key - (int)div_by(key, a.by_page) * a.c.page_size;
  f.at = page * a.c.page_stride + in * a.c.token_stride + p.head * a.c.head_stride + (threadIdx.x & 3) * 4;
  f.scale_at = ((int64_t)page * a.c.n_kv_heads + p.head) * a.c.page_size + in;
  generic_page(a, q, table, kt + 1, f);
}
template <int FORMAT, int ND>
__device__ __forceinline__ void generic_load(const PagedArgs& a, const void* values, const float* scales, GenericShare<ND>& f) {
  const bool there = f.at >= 0;
  f.scale = 1.f;
  if (FORMAT == KEEP_CACHE_FP8 || FORMAT == KEEP_CACHE_INT8) f.scale = scales[there ? f.scale_at : 0];
  const int64_t at = there ? f.at : 0;  // (a place that may be read)
#pragma unroll
  for (int j = 0; j < ND; ++j) f.raw[j] = load_raw<FORMAT>(values, at + min(16 * j, a.c.head_dim - 16));
}
// ... to LDS; returns whether all are finite
template <int FORMAT, int ND>
__device__ __forceinline__ bool generic_store(float* tile, int head_dim, const GenericShare<ND>& f) {
  float* to = tile + (threadIdx.x >> 2) * (16 * ND + 4) + (threadIdx.x & 3) * 4;
  bool ok = true;
#pragma unroll
  for (int j = 0; j < ND; ++j) {
    const bool there = f.at >= 0 && 16 * j < head_dim;
    const f32x4 u = value_of<FORMAT>(f.raw[j], f.scale), v = there ? u : f32x4{0.f, 0.f, 0.f, 0.f};
    ok = ok && finite4(v);
    *reinterpret_cast<f32x4*>(to + 16 * j) = v;
  }
  return ok;
}

// Any types, head_dim a multiple of 16 up to 16 * ND.  A worker's tile is 16 RB query rows and 64 keys; each of the four waves takes
// 16 of the keys for all rows, with statistics and output of its own, added at a job's end.  S^T = K . Q^T leaves a lane one
// query row (lane % 16) of each 16 and four keys (4 (lane / 16) + r), which is the operand that O^T = V^T . P^T wants from it in
// step r: the probabilities never leave their registers.  Rows of K and V in LDS are padded by four values, so that both operand
// reads meet all banks.  V is on its way to registers while the scores are formed, the next tile's K during the second product.
// Many rows: the fp32 matrix instruction is the bound, at half to two thirds of its rate (chunks of up to 2000 tokens over up to
// 16k, heads of 80: 90 TFLOP/s, 128: 72, over an 8-bit cache 98; a large product 154): the barriers of a tile, which two waves
// per SIMD do not hide.  Few rows: HBM (64 tokens over up to 8k fp32 keys 359 us, 5.5 TB/s; one over 33k 65 us).  Staged without
// the loads ahead, with an index for every value: 24 TFLOP/s and 2.1 TB/s.
template <int FORMAT, int ND, int RB>
__global__ void __launch_bounds__(256, ND <= 8 ? 2 : 1) k_paged_generic(PagedArgs a) {
  constexpr int TR = 16 * RB;
  extern __shared__ __attribute__((aligned(16))) float lds[];
  __shared__ int odd[2];  // some value of the tile (by turns) is not finite
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int dh = a.c.head_dim, nd = dh / 16;
  constexpr int stride = 16 * ND + 4;
  // The workgroups of an XCD (blockIdx % 8) take neighbouring runs: one head's tiles read the same keys from its L2
  const int worker = (blockIdx.x & 7) * (PAGED_WORKERS / 8) + (blockIdx.x >> 3);
  PagedSeq q;
  PagedPlace p = paged_place<TR, GT_KEYS>(a, worker, reinterpret_cast<uint64_t*>(lds), q);
  if (tid == 0) a.rec[worker].last = 0;
  if (p.begin >= p.end) return;
  float* sk = lds;
  float* sv = lds + GT_KEYS * stride;
  float* sml = sv + GT_KEYS * stride;  // [2][4 waves][TR]
  for (uint64_t at = p.begin;;) {
    const PagedPart part = paged_part<TR, GT_KEYS>(a, p, q, at);
    if (part.u0 == part.u1) break;  // (the run's last step)
    const int32_t* table = a.table + (int64_t)p.seq * a.max_pages;
    const int kt1 = part.first + part.u1;
    GenericShare<ND> next;
    generic_page(a, q, table, part.first + part.u0, next);
    int pos[RB], lo[RB];
    f32x4 qf[RB][ND], acc[RB][ND];
    float m[RB], l[RB];
    int ln = lane;
    asm volatile("" : "+v"(ln));  // (what follows from it is formed in every job, not kept in registers)
    const int col = ln & 15, g = ln >> 4;
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      const int x = p.tile * TR + 16 * b + col;
      const bool valid = x < q.rows * a.rep;
      const int token = valid ? (int)div_by(x, a.by_rep) : 0;
      const int head = p.head * a.rep + (valid ? x - token * a.rep : 0);
      pos[b] = valid ? q.len - q.rows + token : -1;
      lo[b] = paged_from(pos[b], a.window);
      const int64_t q_at = (int64_t)(q.row0 + token) * a.q_stride + (int64_t)head * dh;
      // (behind the head's width: zeros, read from a place that may be read)
      if (a.dtype == KEEP_F32) {
#pragma unroll
        for (int i = 0; i < ND; ++i)
          qf[b][i] = value_of<KEEP_CACHE_F32>(load_raw<KEEP_CACHE_F32>(a.q, q_at + min(g * 4 * ND + 4 * i, dh - 4)), 1.f);
      } else {
#pragma unroll
        for (int i = 0; i < ND; ++i)
          qf[b][i] = value_of<KEEP_CACHE_BF16>(load_raw<KEEP_CACHE_BF16>(a.q, q_at + min(g * 4 * ND + 4 * i, dh - 4)), 1.f);
      }
#pragma unroll
      for (int i = 0; i < ND; ++i) {
        if (g * 4 * ND + 4 * i >= dh) qf[b][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        acc[b][i] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      m[b] = -INFINITY;
      l[b] = 0.f;
    }
    generic_locate(a, p, q, table, part.first + part.u0, next);
    generic_load<FORMAT>(a, a.c.k, a.c.k_scale, next);
    __syncthreads();  // the LDS of the division, or of the job before, has been read
    if (tid == 0) odd[0] = odd[1] = 0;
    int min_pos, max_lo;  // over the tile's rows
    {
      const int x1 = min(q.rows * a.rep, (p.tile + 1) * TR) - 1;
      min_pos = q.len - q.rows + (int)div_by(p.tile * TR, a.by_rep);
      max_lo = paged_from(q.len - q.rows + (int)div_by(x1, a.by_rep), a.window);
    }
    // One key tile; MASKED: some row does not see some key of it
    const auto tile = [&](int kt, auto masked_type) __attribute__((always_inline)) {
      constexpr bool MASKED = decltype(masked_type)::value;
      const int turn = (kt - part.first - part.u0) & 1;
      generic_store<FORMAT>(sk, dh, next);
      __syncthreads();
      generic_load<FORMAT>(a, a.c.v, a.c.v_scale, next);
      const float* wk = sk + (wave * 16 + col) * stride + g * 4 * ND;
      f32x4 s[RB];
#pragma unroll
      for (int b = 0; b < RB; ++b) s[b] = f32x4{0.f, 0.f, 0.f, 0.f};
      f32x4 ahead = *reinterpret_cast<const f32x4*>(wk);
#pragma unroll
      for (int i = 0; i < ND; ++i) {
        const f32x4 k = ahead;
        if (i + 1 < ND) ahead = *reinterpret_cast<const f32x4*>(wk + 4 * i + 4);
        __builtin_amdgcn_sched_barrier(0);  // (one operand ahead: all of them would push registers out to memory)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int b = 0; b < RB; ++b) s[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], qf[b][i][e], s[b], 0, 0, 0);
      }
      const int key0 = kt * GT_KEYS + wave * 16;
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int key = key0 + 4 * g + r;
          s[b][r] = !MASKED || (key <= pos[b] && key >= lo[b]) ? s[b][r] * a.scale_log2e : -INFINITY;
          top = fmaxf(top, s[b][r]);
        }
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m_new = fmaxf(m[b], top), m_ref = m_new == -INFINITY ? 0.f : m_new;
        if (__ballot(m_new != m[b])) {
          const float alpha = __builtin_amdgcn_exp2f(m[b] - m_ref);
          l[b] *= alpha;
#pragma unroll
          for (int i = 0; i < ND; ++i) acc[b][i] *= alpha;
          m[b] = m_new;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[b][r] = __builtin_amdgcn_exp2f(s[b][r] - m_ref);
          l[b] += s[b][r];
        }
      }
      const bool ok = generic_store<FORMAT>(sv, dh, next);
      if (MASKED && !ok) odd[turn] = 1;
      __syncthreads();
      if (tid == 0) odd[turn ^ 1] = 0;
      if (kt + 1 < kt1) {
        generic_locate(a, p, q, table, kt + 1, next);
        generic_load<FORMAT>(a, a.c.k, a.c.k_scale, next);
      }
      const float* wv = sv + (wave * 16) * stride;
      if (!MASKED || !odd[turn]) {
        constexpr int SOME = ND < 8 ? ND : 4;
        float ahead_v[SOME];
#pragma unroll
        for (int i = 0; i < SOME; ++i) ahead_v[i] = wv[4 * g * stride + 16 * i + col];
#pragma unroll
        for (int n = 0; n < 4 * ND / SOME; ++n) {
          const int r = n * SOME / ND, i0 = n * SOME % ND, n1 = n + 1, r1 = n1 * SOME / ND, i1 = n1 * SOME % ND;
          float v[SOME];
#pragma unroll
          for (int i = 0; i < SOME; ++i) {
            v[i] = ahead_v[i];
            if (r1 < 4) ahead_v[i] = wv[(4 * g + r1) * stride + 16 * (i1 + i) + col];
          }
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int i = 0; i < SOME; ++i)
#pragma unroll
            for (int b = 0; b < RB; ++b)
              acc[b][i0 + i] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[i], s[b][r], acc[b][i0 + i], 0, 0, 0);
        }
      } else {
        // a product with a probability of zero would carry infinities and NaN to rows that do not see the key
#pragma unroll 1
        for (int j = 0; j < 16; ++j) {
          float pj[RB];
#pragma unroll
          for (int b = 0; b < RB; ++b)
            pj[b] = __shfl(j & 2 ? j & 1 ? s[b][3] : s[b][2] : j & 1 ? s[b][1] : s[b][0], (j >> 2) * 16 + col, 64);
#pragma unroll
          for (int i = 0; i < ND; ++i) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(wv + j * stride + 16 * i + 4 * g);
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[b][i][e] += key0 + j <= pos[b] && key0 + j >= lo[b] ? pj[b] * v[e] : 0.f;
            __builtin_amdgcn_sched_barrier(0);  // (one read at a time: this path must not cost the other registers)
          }
        }
      }
    };
    // Two loops, so that what masks need takes no registers from the tiles without: they are nearly all of them
    const auto is_masked = [&](int kt) { return kt * GT_KEYS + GT_KEYS - 1 > min_pos || kt * GT_KEYS < max_lo; };
    for (int kt = part.first + part.u0; kt < kt1;) {
      for (; kt < kt1 && !is_masked(kt); ++kt) tile(kt, std::false_type{});
      for (; kt < kt1 && is_masked(kt); ++kt) tile(kt, std::true_type{});
    }

    // ---- the four waves' parts, in their order
    __syncthreads();
    float* so = lds;  // [4 waves][dh / 4][TR][4]
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      l[b] += __shfl_xor(l[b], 16, 64);
      l[b] += __shfl_xor(l[b], 32, 64);
      if (g == 0) sml[wave * TR + 16 * b + col] = m[b], sml[(4 + wave) * TR + 16 * b + col] = l[b];
#pragma unroll
      for (int i = 0; i < ND; ++i)
        if (i < nd) *reinterpret_cast<f32x4*>(so + ((wave * (dh / 4) + 4 * i + g) * TR + 16 * b + col) * 4) = acc[b][i];
    }
    __syncthreads();
    paged_finish<TR>(a, p, q, part, worker, so, sml);
    at += part.steps;
    if (at >= p.end) break;
    paged_next<TR>(a, p, q);
  }
}

// The parts of a job that was cut, joined in the order of their keys.  Workgroup x takes the x-th job that a worker left a record
// of, and `groups` times 16 of the output's dimensions (blockIdx.y).  Lanes lie along query rows, then along parts, and as many
// waves as there are to spare for 16 dimensions along parts again, each lane with a running maximum and sum of its own, so that all
// loads are independent of one another; a butterfly adds the lanes of a row, LDS the waves.
// A chain of three reads that each wait for the one before (records, record, parts) bounds it.  8 jobs of 64 parts of 5 rows: 17 us
// more with the parts along 8 lanes and two passes over them, 8 more with 4096 workgroups of which nearly all find no record, 3
// more with a wave for all of a job's parts.  512 jobs: 8 us, 10 with registers for one workgroup per CU only.
template <int TR>
__global__ void __launch_bounds__(512, 4) k_paged_join(PagedArgs a, int groups) {
  constexpr int RB = TR < 64 ? TR : 64;  // rows side by side in a wave
  __shared__ float s_m[8][RB], s_l[8][RB];
  __shared__ f32x4 s_o[8][4][RB];
  __shared__ int s_count[8], s_w0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (gridDim.x == PAGED_WORKERS) {  // a workgroup for every worker: no need to count
    if (a.rec[blockIdx.x].last == 0) return;
    if (threadIdx.x == 0) s_w0 = blockIdx.x;
    __syncthreads();
  } else {
    static_assert(PAGED_WORKERS == 512, "a thread looks at one record");
    const bool is = a.rec[threadIdx.x].last != 0;
    const uint64_t some = __ballot(is);
    if (lane == 0) s_count[wave] = __popcll(some);
    if (threadIdx.x == 0) s_w0 = -1;
    __syncthreads();
    int rank = __popcll(some & ((1ull << lane) - 1));
    for (int w = 0; w < wave; ++w) rank += s_count[w];
    if (is && rank == (int)blockIdx.x) s_w0 = threadIdx.x;
    __syncthreads();
  }
  const int w0 = s_w0;
  if (w0 < 0) return;
  const PagedRecord r = a.rec[w0];
  const int quads = a.c.head_dim / 4, n = r.last - w0 + 1;
  int rb = 1, along = 1;  // rows in a wave; waves along the parts
  while (rb < min(r.n, RB)) rb *= 2;
  while (2 * along * groups <= 8) along *= 2;
  const int lanes = 64 / rb, part0 = (wave & (along - 1)) * lanes + lane / rb, step = along * lanes;
  for (int g0 = 0; g0 < groups; g0 += 8 / along) {
    const int q0 = ((int)blockIdx.y * groups + g0 + wave / along) * 4;
    const bool dims = g0 + wave / along < groups && q0 < quads;
    for (int base = 0; base < r.n; base += rb) {
      const int row = base + (lane & (rb - 1));
      const bool valid = dims && row < r.n;
      float m = -INFINITY, l = 0.f;
      f32x4 o[4] = {};
      if (valid) {
#pragma unroll 4
        for (int i = part0; i < n; i += step) {
          const int64_t slot = i == 0 ? 2 * w0 + 1 : 2 * (w0 + i);
          const float mi = a.part_ml[slot * 2 * TR + row], li = a.part_ml[(slot * 2 + 1) * TR + row];
          f32x4 v[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const f32x4*>(a.part_o + ((slot * quads + q0 + j) * TR + row) * 4);
          const float m_new = fmaxf(m, mi), ref = m_new == -INFINITY ? 0.f : m_new;
          const float old = __builtin_amdgcn_exp2f(m - ref), now = __builtin_amdgcn_exp2f(mi - ref);
          l = l * old + li * now;
#pragma unroll
          for (int j = 0; j < 4; ++j) o[j] = o[j] * old + (now == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : v[j] * now);
          m = m_new;
        }
      }
      const float m0 = m;
      for (int s = rb; s < 64; s <<= 1) m = fmaxf(m, __shfl_xor(m, s, 64));
      const float scale = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m0 - m);
      l *= scale;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] *= scale;
      for (int s = rb; s < 64; s <<= 1) {
        l += __shfl_xor(l, s, 64);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[j][e] += __shfl_xor(o[j][e], s, 64);
      }
      if (along > 1) {
        __syncthreads();  // (the sums before have been read)
        if (lane < rb) {
          s_m[wave][lane] = m, s_l[wave][lane] = l;
#pragma unroll
          for (int j = 0; j < 4; ++j) s_o[wave][j][lane] = o[j];
        }
        __syncthreads();
        if ((wave & (along - 1)) != 0 || lane >= rb) continue;
        for (int w = wave; w < wave + along; ++w) m = fmaxf(m, s_m[w][lane]);
        l = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int w = wave; w < wave + along; ++w) {
          const float f = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(s_m[w][lane] - m);
          l += s_l[w][lane] * f;
#pragma unroll
          for (int j = 0; j < 4; ++j) o[j] += f == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : s_o[w][j][lane] * f;
        }
      }
      if (!valid || lane >= rb) continue;
      const int x = r.x0 + row, token = (int)div_by(x, a.by_rep), head = r.head * a.rep + x - token * a.rep;
      const int64_t o_at = (int64_t)(r.row0 + token) * a.out_stride + (int64_t)head * a.c.head_dim + q0 * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (l != 0.f) o[j] /= l;
        if (a.dtype == KEEP_F32)
          *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + o_at + 4 * j) = o[j];
        else
          *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + o_at + 4 * j) =
              make_uint2(pack_bf16x2(o[j][0], o[j][1]), pack_bf16x2(o[j][2], o[j][3]));
      }
      if (q0 == 0 && a.lse) a.lse[(int64_t)(r.row0 + token) * a.n_q_heads + head] = 0.6931471805599453f * (m + log2f(l));
    }
  }
}

uint64_t part_bytes(int tr, int dh) { return (uint64_t)2 * PAGED_WORKERS * tr * (dh + 2) * sizeof(float); }
// caches that paged_attn_mfma.hip has a kernel for (with bf16 queries); offsets in 16 bytes fit 32 bits
bool has_mfma(const keep_paged_cache* c) {
  const int64_t span = (int64_t)(c->n_pages - 1) * c->page_stride + (int64_t)(c->n_kv_heads - 1) * c->head_stride +
                       (int64_t)(c->page_size - 1) * c->token_stride + c->head_dim;
  return c->format != KEEP_CACHE_F32 && (c->head_dim == 64 || c->head_dim == 128 || c->head_dim == 256) &&
         span * format_size(c->format) < (int64_t)64 << 30;
}
constexpr uint64_t REC_BYTES = (PAGED_WORKERS * sizeof(PagedRecord) + 255) & ~(uint64_t)255;

}  // namespace

template <int FORMAT, int ND, int RB>
static void launch_generic(const PagedArgs& a, hipStream_t s) {
  // tiles (or the waves' outputs, which need no more) and statistics; the division of the work before that
  const size_t lds = std::max<size_t>(((size_t)2 * GT_KEYS * (16 * ND + 4) + 8 * 16 * RB) * sizeof(float), (size_t)8 * (a.n_seqs + 260));
  static std::atomic<uint64_t> done{0};
  set_max_dyn_smem_once(done, reinterpret_cast<const void*>(k_paged_generic<FORMAT, ND, RB>), 150 * 1024);
  hipLaunchKernelGGL((k_paged_generic<FORMAT, ND, RB>), dim3(PAGED_WORKERS), dim3(256), lds, s, a);
  launch_paged_join(a, 16 * RB, s);
}
// Whether tiles of 32 query rows have the registers: with fp32 keys of 128 they would spill (us on tiles of 16 / 32: one sequence of
// 33k keys with 20 rows 87 / 113, eight chunks 8193 / 8764, but 64 sequences of up to 8k keys with 20 rows 630 / 587).
constexpr bool paged_wide_tiles(int format, int head_dim) { return head_dim <= (format == KEEP_CACHE_F32 ? 80 : 128); }

template <int FORMAT>
static void launch_generic(const PagedArgs& a, int rows, hipStream_t s) {
  const int dh = a.c.head_dim;
  // (tiles of 16 rows where there are none of 32: they and their join fit a workspace laid out for 32)
  if (rows == 32 && paged_wide_tiles(FORMAT, dh)) {
    if (dh <= 64) return launch_generic<FORMAT, 4, 2>(a, s);
    if (dh <= 80) return launch_generic<FORMAT, 5, 2>(a, s);
    if constexpr (paged_wide_tiles(FORMAT, 128)) return launch_generic<FORMAT, 8, 2>(a, s);
  }
  return dh <= 64    ? launch_generic<FORMAT, 4, 1>(a, s)
         : dh <= 80  ? launch_generic<FORMAT, 5, 1>(a, s)
         : dh <= 128 ? launch_generic<FORMAT, 8, 1>(a, s)
                     : launch_generic<FORMAT, 16, 1>(a, s);
}

void launch_paged_generic(const PagedArgs& a, int rows, hipStream_t s) {
  switch (a.c.format) {
    case KEEP_CACHE_F32: return launch_generic<KEEP_CACHE_F32>(a, rows, s);
    case KEEP_CACHE_BF16: return launch_generic<KEEP_CACHE_BF16>(a, rows, s);
    case KEEP_CACHE_FP8: return launch_generic<KEEP_CACHE_FP8>(a, rows, s);
    default: return launch_generic<KEEP_CACHE_INT8>(a, rows, s);
  }
}

void launch_paged_join(const PagedArgs& a, int rows, hipStream_t s) {
  // no more jobs than tiles, and few workgroups share the dimensions of few jobs
  const int64_t tiles = (a.n_rows * (int64_t)a.rep / rows + a.n_seqs) * a.c.n_kv_heads;
  const int jobs = (int)std::min<int64_t>(PAGED_WORKERS, tiles), all = a.c.head_dim / 16;
  const int groups = (all + std::max(1, 256 / jobs) - 1) / std::max(1, 256 / jobs);
  const auto kernel = rows == 16 ? k_paged_join<16> : rows == 32 ? k_paged_join<32> : k_paged_join<128>;
  hipLaunchKernelGGL(kernel, dim3(jobs, (all + groups - 1) / groups), dim3(512), 0, s, a, groups);
}

}  // namespace keep

using namespace keep;

extern "C" uint64_t keep_paged_attention_workspace_bytes(const keep_paged_cache* cache, int32_t n_q_heads, int32_t n_seqs) {
  if (check_cache(cache, "keep_paged_attention_workspace_bytes") != KEEP_OK) return 0;
  if (n_q_heads < 1 || n_q_heads % cache->n_kv_heads || n_seqs < 0 || n_seqs > KEEP_PAGED_MAX_SEQS) return 0;
  return REC_BYTES + part_bytes(has_mfma(cache) && cache->head_dim <= 128 ? 128 : 32, cache->head_dim);
}

extern "C" keep_status keep_paged_attention(const keep_paged_attention_desc* d, const keep_paged_cache* cache, const void* q,
                                            const int32_t* q_start, const int32_t* kv_len, const int32_t* page_table, void* out,
                                            float* lse, void* workspace, uint64_t workspace_bytes, void* stream) {
  const char* me = "keep_paged_attention";
  if (!d) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: desc is NULL", me);
  const keep_status st = check_cache(cache, me);
  if (st != KEEP_OK) return st;
  if (!is_dtype(d->dtype)) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: unknown dtype %d", me, d->dtype);
  if (d->n_seqs < 0 || d->n_rows < 0 || d->window < 0)
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: n_seqs, n_rows or window is negative", me);
  if (d->n_seqs > KEEP_PAGED_MAX_SEQS)
    return serve_fail(KEEP_ERR_SHAPE, "%s: more than %d sequences", me, KEEP_PAGED_MAX_SEQS);
  if (d->n_q_heads < 1 || d->n_q_heads % cache->n_kv_heads)
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: n_q_heads %d is no multiple of n_kv_heads %d", me, d->n_q_heads,
                      cache->n_kv_heads);
  if (d->max_pages < 1 || (int64_t)d->max_pages * cache->page_size > INT32_MAX - 1023)
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: max_pages must be at least 1 and max_pages * page_size at most 2^31 - 1024", me);
  if (!isfinite(d->scale)) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: scale is not finite", me);
  const int size = dtype_size(d->dtype);
  const int64_t width = (int64_t)d->n_q_heads * cache->head_dim;
  if (d->n_rows * (int64_t)(d->n_q_heads / cache->n_kv_heads) > INT32_MAX - 1024)
    return serve_fail(KEEP_ERR_SHAPE, "%s: too many query rows", me);
  if (d->q_stride < width || d->out_stride < width || d->q_stride * size % 16 || d->out_stride * size % 16)
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: a row stride must hold the row's %lld values and be a multiple of 16 bytes", me,
                      (long long)width);
  if (d->n_seqs == 0 || d->n_rows == 0) return KEEP_OK;
  if (!q || !q_start || !kv_len || !page_table || !out || !workspace)
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: q / q_start / kv_len / page_table / out / workspace is NULL", me);
  if (!aligned16(q) || !aligned16(out) || reinterpret_cast<uintptr_t>(workspace) % 256)
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: q, out or workspace is not aligned", me);
  if (overlaps({q, d->q_stride, width}, {out, d->out_stride, width}, d->n_rows, size))
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: q and out overlap", me);
  if (workspace_bytes < keep_paged_attention_workspace_bytes(cache, d->n_q_heads, d->n_seqs))
    return serve_fail(KEEP_ERR_WORKSPACE, "%s: workspace of %llu bytes is too small", me, (unsigned long long)workspace_bytes);
  PagedArgs a{};
  a.c = *cache;
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.q_start = q_start;
  a.kv_len = kv_len;
  a.table = page_table;
  a.q_stride = d->q_stride;
  a.out_stride = d->out_stride;
  a.n_seqs = d->n_seqs;
  a.n_rows = d->n_rows;
  a.n_q_heads = d->n_q_heads;
  a.rep = d->n_q_heads / cache->n_kv_heads;
  a.max_pages = d->max_pages;
  a.window = d->window;
  a.capacity = d->max_pages * cache->page_size;
  a.dtype = d->dtype;
  a.scale_log2e = (d->scale == 0.f ? 1.f / sqrtf((float)cache->head_dim) : d->scale) * 1.4426950408889634f;
  a.by_page = fast_div((uint32_t)cache->page_size);
  a.by_rep = fast_div((uint32_t)a.rep);
  char* ws = static_cast<char*>(workspace);
  a.rec = reinterpret_cast<PagedRecord*>(ws);
  a.part_ml = reinterpret_cast<float*>(ws + REC_BYTES);
  if (!format_scaled(cache->format)) a.c.k_scale = a.c.v_scale = nullptr;
  // The bf16 matrix instruction where it has a kernel, in tiles of 16, 32 or 128 query rows by what a sequence brings on average.
  // us on tiles of 16 / 32 / 128 for 30, 60 and 125 rows per sequence, 64 ragged sequences of up to 8k keys in bf16: 331 / 213 /
  // 260, 629 / 351 / 284, 1207 / 671 / 303 (fp8: 184 / 143 / 237, 340 / 233 / 260); one sequence of 33k keys: 55 / 50 / 58,
  // 59 / 56 / 64, 89 / 67 / 75.  Up to 16 rows a tile of 32 has nothing to gain.
  const bool mfma = d->dtype == KEEP_BF16 && has_mfma(cache);
  const int64_t mean = (d->n_rows * (int64_t)a.rep + d->n_seqs - 1) / d->n_seqs;
  int rows = mean <= 16 ? 16 : 32;
  if (mfma && cache->head_dim == 256) {
    // (heads of 256: a workgroup per CU with bf16 keys or 32 rows.  us on tiles of 16 / 32: 64 sequences of up to 8k 8-bit keys with
    // 32 rows 58 / 104, eight chunks 937 / 1432; bf16, 32, 128, 512 and 2048 rows 99 / 122, 262 / 257, 931 / 819, 3699 / 3286,
    // one sequence of 33k keys with 512 and 8000 rows 119 / 134, 2462 / 1257)
    rows = cache->format == KEEP_CACHE_BF16 && mean > 512 ? 32 : 16;
  } else if (mfma) {
    if (mean > 48) rows = 128;
  } else {
    // The fp32 kernel has no tiles of 32 rows where their registers do not fit (paged_wide_tiles), and where such tiles would not
    // give every worker two units, smaller ones end sooner (three short sequences with heads of 64: 10.4 us instead of 12.6).
    // Else us on tiles of 16 / 32, 64 sequences of up to 8k 8-bit keys with 20 and 60 rows: 449 / 357, 883 / 698; one of 33k with
    // 125 rows: 242 / 201; eight chunks of up to 2000 tokens: 7671 / 6052.
    const double units = (d->n_rows * (double)a.rep / 32 + d->n_seqs) * cache->n_kv_heads * (a.capacity / 64 + 1);
    if (!paged_wide_tiles(cache->format, cache->head_dim) || units < 2 * PAGED_WORKERS) rows = 16;
  }
  a.part_o = a.part_ml + (size_t)2 * PAGED_WORKERS * 2 * rows;
  if (mfma)
    launch_paged_mfma(a, rows, static_cast<hipStream_t>(stream));
  else
    launch_paged_generic(a, rows, static_cast<hipStream_t>(stream));
  return launched(me);
}
