// Attention over pages on the bf16 matrix instruction: bf16 queries, heads of 64, 128 or 256, a bf16 or 8-bit cache.
//
// k_paged_few: tiles of 16 or 32 query rows (one to a few tokens with their heads), where the keys are read once for few rows and
// memory is the bound.  Each of a workgroup's four waves streams key slices of its own (32 of a unit's 128 keys) through its own
// part of LDS, without barriers: K and V arrive by loads that go straight to LDS as they are stored, the next slice's K is
// requested as soon as this one's has been read and the same for V, so that a wave always has loads in flight; two workgroups
// per CU keep some 100 KB on their way.
//
// Scores are formed transposed, S^T = K . Q^T (16x16x32): a lane owns a query row (lane % 16) and keys 4 (lane / 16) + r of both
// 16-key blocks, which as they stand are the operand of O^T = V^T . P^T; its V^T operand comes from the transposing LDS
// reads (ds_read_b64_tr_b16, _tr_b8).  8-bit codes become bf16 exactly (at most 8 significant bits) when they are read as
// operands; a key's scale multiplies its scores, a value's scale its probability, in binary32.  Probabilities (with the
// value's scale) are rounded to bf16 for the product, the row sums are taken before that.
//
// 64 sequences of one token with 40 / 8 heads of 128 over up to 8k keys in fp8 (512 MB): 111 us, 4.6 TB/s (and 8 for the join) where a
// copy reaches 4.7; one token over 33k bf16 keys (135 MB): 33 us, 4.1 TB/s (and 9).  The first kernel, on the fp32 matrix
// instruction with staging behind barriers, took 940 and 167.
//
// k_paged_many: tiles of 128 query rows, 32 per wave, over key tiles of 64 that the workgroup shares in LDS (two of them: the
// next arrives while one is used), where the matrix instruction and the exponentials are the bound.  32x32x16: a lane owns a
// query row (lane % 32) and half of the tile's keys, and again S^T = K . Q^T leaves the operand of O^T = V^T . P^T.
// 8-bit codes become bf16 on their way into LDS, once for the four waves.
// Eight chunks of 100 to 2000 tokens over up to 16k keys, 28 / 4 heads of 128, bf16 (589 GFLOP): 765 us and 23 for the join, 792
// and 743 TFLOP/s a call, where a large product reaches 1419; 256 tokens over 33k int8 keys, 40 / 8 heads: 263 and 16, 269 a
// call, 640 TFLOP/s (bf16 15 % more).  Cards differ: 256 to 276 and 762 to 810 a call.  Exponentials and conversions share the
// SIMD with the products, and 32 rows per wave feed each K and V operand to one product only.
#include <type_traits>

#include "paged_attn.h"

namespace keep {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(2))) int i32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
using f32x4 = paged_f32x4;
typedef s16x4 __attribute__((address_space(3))) * lds_s16x4;
typedef i32x2 __attribute__((address_space(3))) * lds_i32x2;
typedef char __attribute__((address_space(3))) * lds_char;

__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(lds_char)p; }

// 16 (4) bytes per lane from global memory to LDS address `to` + 16 (4) * lane.  Written out because the compiler would wait
// for these loads before every later LDS read; vm_wait below says which have landed.  (m0 holds the LDS address; nothing that
// the compiler makes of these kernels reads it.)
__device__ __forceinline__ void load_lds16(const void* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to) : "memory");
}
__device__ __forceinline__ void load_lds4(const void* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(from), "s"(to) : "memory");
}
template <int N>
__device__ __forceinline__ void vm_wait() {  // all but the N youngest vector loads have landed
  static_assert(N >= 0 && N < 64, "the counter has six bits");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void lds_wait() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Over the four lanes of a query row (lane % 16)
__device__ __forceinline__ float row_max(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float row_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// Eight codes as bf16 numbers
template <int FMT>
__device__ __forceinline__ bf16x8 codes8(uint32_t lo, uint32_t hi) {
  u32x4 r;
  if constexpr (FMT == KEEP_CACHE_FP8) {
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t w = i ? hi : lo;
      r[2 * i] = pack_bf16x2((float)(int8_t)w, (float)(int8_t)(w >> 8));
      r[2 * i + 1] = pack_bf16x2((float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24));
    }
  }
  return __builtin_bit_cast(bf16x8, r);
}

// Where the 16-byte chunk c of a slice's row lies inside the row.  LDS serves 256 bytes at a time: a K read 16 rows (lane % 16) at one
// chunk, a V read half a wave: eight rows of two chunks (bf16), or 16 rows (4 g + j and 16 + 4 g + j, two g) of one chunk.
// CH: chunks per row; 16 / CH rows share a stretch of 256 bytes, the chunks of those that lie at the same place move apart.
template <int CH>
__device__ __forceinline__ int k_chunk(int row, int c) {
  return CH >= 16 ? c ^ (row & 15) : CH == 8 ? c ^ ((row >> 1) & 7) : c ^ ((row >> 2) & 3);
}
template <int CH, bool WIDE>  // WIDE: bf16
__device__ __forceinline__ int v_chunk(int row, int c) {
  if (WIDE) return CH >= 16 ? c ^ (2 * (row & 7)) : c ^ (2 * ((row >> 1) & 3));
  if (CH == 16) return c ^ ((row & 7) | ((row >> 1) & 8));
  return CH == 8 ? c ^ (((row >> 1) & 3) | ((row >> 2) & 4)) : c ^ (((row >> 2) & 1) | ((row >> 3) & 2));
}

constexpr int SLICE = 32, UNIT = 4 * SLICE;  // keys of a wave's slice, of a unit
constexpr int TABLE = 1024;                  // page table entries held in LDS at a time

template <int DH, int FMT, int RB>
struct Few {
  static constexpr bool WIDE = FMT == KEEP_CACHE_BF16;
  static constexpr int TR = 16 * RB;
  static constexpr int ROW = DH * (WIDE ? 2 : 1), CH = ROW / 16;  // bytes and chunks of a key
  static constexpr int PER = 64 / CH, NI = SLICE / PER;           // rows of a load, loads of a slice
  static constexpr int BYTES = SLICE * ROW;
  static constexpr int HELD = TR * DH * 4 > 16384 ? TR * DH * 4 : 16384;            // bytes of a wave: its slices, at the end its output
  static constexpr int NS = 2 * BYTES < HELD ? HELD / (2 * BYTES) : 1;              // slices in flight
  static constexpr int NK = NI + (WIDE ? 0 : 1), NV = NI;         // loads of a slice's K (with the scales) and V
  static constexpr int WAVE = NS * (2 * BYTES + (WIDE ? 0 : 256));
  static constexpr int ML = 4 * WAVE, TBL = ML + 8 * TR * 4, LDS = TBL + TABLE * 4;
  static_assert(4 * TR * DH * 4 <= 4 * WAVE, "the waves' outputs lie where the slices did");
};

template <int DH, int FMT, int RB>
__global__ void __launch_bounds__(256, (Few<DH, FMT, RB>::LDS > 80 * 1024 ? 1 : 2)) k_paged_few(PagedArgs a) {
  using F = Few<DH, FMT, RB>;
  constexpr int TR = F::TR, ROW = F::ROW, CH = F::CH, NS = F::NS, DT = DH / 16, KS = DH / 32;
  extern __shared__ __attribute__((aligned(256))) char lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, g = lane >> 4;
  // The workgroups of an XCD (blockIdx % 8) take neighbouring runs: one head's tiles read the same keys from its L2
  const int worker = (blockIdx.x & 7) * (PAGED_WORKERS / 8) + (blockIdx.x >> 3);
  PagedSeq q;
  PagedPlace p = paged_place<TR, UNIT>(a, worker, reinterpret_cast<uint64_t*>(lds), q);
  if (tid == 0) a.rec[worker].last = 0;
  if (p.begin >= p.end) return;
  char* ring = lds + wave * F::WAVE;  // [NS] K slices, [NS] V slices, [NS] scales (32 of keys, 32 of values)
  const uint32_t ring_at = __builtin_amdgcn_readfirstlane(lds_address(ring));
  float* sml = reinterpret_cast<float*>(lds + F::ML);
  int32_t* tbl = reinterpret_cast<int32_t*>(lds + F::TBL);
  const char* k_base = static_cast<const char*>(a.c.k);
  const char* v_base = static_cast<const char*>(a.c.v);
  const int block_units = (int)max((int64_t)1, min((int64_t)1 << 20, (int64_t)(TABLE - 2) * a.c.page_size / UNIT));

  for (uint64_t at = p.begin;;) {
    const PagedPart part = paged_part<TR, UNIT>(a, p, q, at);
    if (part.u0 == part.u1) break;  // (the run's last step)
    const int first = part.first, u1 = part.u1;
    // ---- this lane's query rows
    int pos[RB], lo[RB];
    bf16x8 qf[RB][KS];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      const int x = p.tile * TR + b * 16 + col;
      const bool valid = x < q.rows * a.rep;
      const int token = valid ? (int)div_by(x, a.by_rep) : 0;
      pos[b] = valid ? q.len - q.rows + token : -1;
      lo[b] = paged_from(pos[b], a.window);
      const __bf16* qp = static_cast<const __bf16*>(a.q) + (int64_t)(q.row0 + token) * a.q_stride +
                         (int64_t)(p.head * a.rep + (valid ? x - token * a.rep : 0)) * DH;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)  // the dimensions that the K operand of step ks holds
        qf[b][ks] = *reinterpret_cast<const bf16x8*>(qp + (F::WIDE ? ks * 32 + g * 8 : (ks >> 1) * 64 + g * 16 + (ks & 1) * 8));
    }
    int max_pos, min_pos, max_lo;  // over the tile
    {
      const int x1 = min(q.rows * a.rep, (p.tile + 1) * TR) - 1;
      max_pos = q.len - q.rows + (int)div_by(x1, a.by_rep);
      min_pos = q.len - q.rows + (int)div_by(p.tile * TR, a.by_rep);
      max_lo = paged_from(max_pos, a.window);
    }
    f32x4 acc[RB][DT];
    float m[RB], l[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      m[b] = -INFINITY, l[b] = 0.f;
#pragma unroll
      for (int i = 0; i < DT; ++i) acc[b][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int32_t* table = a.table + (int64_t)p.seq * a.max_pages;
    const int64_t head_at = (int64_t)p.head * a.c.head_stride * (F::WIDE ? 2 : 1);

    for (int ub = part.u0; ub < u1; ub += block_units) {
      const int ue = min(u1, ub + block_units);
      const int page0 = (int)div_by((uint32_t)(first + ub) * UNIT, a.by_page);
      const int page1 = (int)div_by((uint32_t)min((int64_t)(first + ue) * UNIT - 1, (int64_t)max(q.len, 1) - 1), a.by_page);
      __syncthreads();  // earlier entries, or the outputs of the job before, have been read
      for (int i = tid; i <= page1 - page0; i += 256) tbl[i] = min(max(table[page0 + i], 0), a.c.n_pages - 1);
      __syncthreads();
      // (the queries, requested before the table, are in registers before the slices' loads begin: the compiler would wait for
      // them, and so for those, in every slice)
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[b][ks]));
      // ---- this wave's slices: keys key0 + UNIT * t, while some row sees them
      const int key0 = (first + ub) * UNIT + wave * SLICE;
      const int n = key0 > max_pos ? 0 : min(ue - ub, (max_pos - key0) / UNIT + 1);
      uint32_t v_off = 0;  // per lane: where key lane % 32 of the youngest requested slice lies, in 16 bytes
      // (What follows from the lane is formed anew in every slice: kept, it would push registers out to memory.)
      const auto request_k = [&](int t) {
        int ln = lane;
        asm volatile("" : "+v"(ln));
        const int key = min(key0 + t * UNIT + (ln & 31), q.len - 1), pg = (int)div_by(key, a.by_page);
        const int page = tbl[pg - page0], in = key - pg * a.c.page_size;
        const uint32_t off = (uint32_t)((page * a.c.page_stride + in * a.c.token_stride) * (F::WIDE ? 2 : 1) / 16);
        const int slot = t % NS;
        if constexpr (!F::WIDE)
          load_lds4((ln < 32 ? a.c.k_scale : a.c.v_scale) + ((int64_t)page * a.c.n_kv_heads + p.head) * a.c.page_size + in,
                    ring_at + 2 * NS * F::BYTES + slot * 256);
#pragma unroll
        for (int i = 0; i < F::NI; ++i) {
          const int row = i * F::PER + ln / CH;
          load_lds16(k_base + head_at + (int64_t)(uint32_t)__shfl((int)off, row, 64) * 16 + k_chunk<CH>(row, ln % CH) * 16,
                     ring_at + slot * F::BYTES + i * 1024);
        }
        return off;
      };
      const auto request_v = [&](int t) {
        const int slot = t % NS;
        int ln = lane;
        asm volatile("" : "+v"(ln));
#pragma unroll
        for (int i = 0; i < F::NI; ++i) {
          const int row = i * F::PER + ln / CH;
          load_lds16(v_base + head_at + (int64_t)(uint32_t)__shfl((int)v_off, row, 64) * 16 + v_chunk<CH, F::WIDE>(row, ln % CH) * 16,
                     ring_at + (NS + slot) * F::BYTES + i * 1024);
        }
      };
      if (n > 0) vm_wait<0>();  // (nothing of the compiler's own is counted below)
      for (int t = 0; t < min(n, NS); ++t) {
        v_off = request_k(t);
        request_v(t);
      }
      // One slice; MASKED: some row does not see some key of it
      const auto slice = [&](int t, auto masked_type) __attribute__((always_inline)) {
        constexpr bool MASKED = decltype(masked_type)::value;
        const int slot = t % NS, kb = key0 + t * UNIT, left = min(NS - 1, n - 1 - t);
        int ln = lane;
        asm volatile("" : "+v"(ln));
        const int col = ln & 15, g = ln >> 4;
        const char* sk = ring + slot * F::BYTES;
        const char* sv = ring + (NS + slot) * F::BYTES;
        const float* scales = reinterpret_cast<const float*>(ring + 2 * NS * F::BYTES + slot * 256);
        // K of this slice has landed; behind it V and `left` whole slices were requested
        switch (left) {
          case 0: vm_wait<F::NV>(); break;
          case 1: vm_wait<NS < 2 ? 0 : F::NV + F::NK + F::NV>(); break;
          case 2: vm_wait<NS < 3 ? 0 : F::NV + 2 * (F::NK + F::NV)>(); break;
          default: vm_wait<NS < 4 ? 0 : F::NV + 3 * (F::NK + F::NV)>(); break;
        }
        f32x4 s[RB][2];
#pragma unroll
        for (int b = 0; b < RB; ++b) s[b][0] = s[b][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kb16 = 0; kb16 < 2; ++kb16) {
          const int row = kb16 * 16 + col;
          if constexpr (F::WIDE) {
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
              const bf16x8 kf = *reinterpret_cast<const bf16x8*>(sk + row * ROW + k_chunk<CH>(row, 4 * ks + g) * 16);
#pragma unroll
              for (int b = 0; b < RB; ++b) s[b][kb16] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[b][ks], s[b][kb16], 0, 0, 0);
            }
          } else {
#pragma unroll
            for (int k2 = 0; k2 < KS / 2; ++k2) {
              const u32x4 c = *reinterpret_cast<const u32x4*>(sk + row * ROW + k_chunk<CH>(row, 4 * k2 + g) * 16);
              const bf16x8 f0 = codes8<FMT>(c[0], c[1]), f1 = codes8<FMT>(c[2], c[3]);
#pragma unroll
              for (int b = 0; b < RB; ++b) {
                s[b][kb16] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f0, qf[b][2 * k2], s[b][kb16], 0, 0, 0);
                s[b][kb16] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f1, qf[b][2 * k2 + 1], s[b][kb16], 0, 0, 0);
              }
            }
          }
        }
        f32x4 k_sc[2], v_sc[2];
        if constexpr (!F::WIDE) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            k_sc[i] = *reinterpret_cast<const f32x4*>(scales + i * 16 + 4 * g) * a.scale_log2e;
            v_sc[i] = *reinterpret_cast<const f32x4*>(scales + 32 + i * 16 + 4 * g);
          }
        }
        lds_wait();  // K and the scales are in registers: their places may be written
        if (t + NS < n) v_off = request_k(t + NS);

        // ---- scores in the log2 domain, running maximum and sum
        bf16x8 pf[RB];
        float pr[RB][8];
#pragma unroll
        for (int b = 0; b < RB; ++b) {
          float top = -INFINITY;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float v = s[b][e >> 2][e & 3];
            if constexpr (F::WIDE)
              v *= a.scale_log2e;
            else
              v *= k_sc[e >> 2][e & 3];
            if constexpr (MASKED) {
              const int key = kb + (e >> 2) * 16 + 4 * g + (e & 3);
              v = key <= pos[b] && key >= lo[b] ? v : -INFINITY;
            }
            pr[b][e] = v;
            top = fmaxf(top, v);
          }
          const float m_new = fmaxf(m[b], row_max(top)), m_ref = m_new == -INFINITY ? 0.f : m_new;
          if (__ballot(m_new != m[b])) {
            const float alpha = __builtin_amdgcn_exp2f(m[b] - m_ref);
            l[b] *= alpha;
#pragma unroll
            for (int i = 0; i < DT; ++i) acc[b][i] *= alpha;
            m[b] = m_new;
          }
          u32x4 pk;
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            float p0 = __builtin_amdgcn_exp2f(pr[b][e] - m_ref), p1 = __builtin_amdgcn_exp2f(pr[b][e + 1] - m_ref);
            l[b] += p0 + p1;
            if constexpr (!F::WIDE) {
              const float v0 = v_sc[e >> 2][e & 3], v1 = v_sc[e >> 2][(e & 3) + 1];
              // (a scale of NaN must not reach rows that do not see the key)
              p0 = MASKED && pr[b][e] == -INFINITY ? 0.f : p0 * v0;
              p1 = MASKED && pr[b][e + 1] == -INFINITY ? 0.f : p1 * v1;
            }
            pr[b][e] = p0, pr[b][e + 1] = p1;
            pk[e >> 1] = pack_bf16x2(p0, p1);
          }
          pf[b] = __builtin_bit_cast(bf16x8, pk);
        }

        // ---- V of this slice has landed; behind it the K requested above and `left` slices of before
        if (t + NS < n) {
          vm_wait<(NS - 1) * (F::NK + F::NV) + F::NK>();
        } else {
          switch (left) {
            case 0: vm_wait<0>(); break;
            case 1: vm_wait<F::NK + F::NV>(); break;
            case 2: vm_wait<NS < 3 ? 0 : 2 * (F::NK + F::NV)>(); break;
            default: vm_wait<NS < 4 ? 0 : 3 * (F::NK + F::NV)>(); break;
          }
        }
        bool odd = false;
        if constexpr (MASKED && FMT != KEEP_CACHE_INT8) {
          // A product with a probability of zero would carry infinities and NaN to rows that do not see the key.
          constexpr uint32_t EXP = F::WIDE ? 0x7f807f80u : 0x7f7f7f7fu;
#pragma unroll 2
          for (int i = lane; i < F::BYTES / 16; i += 64) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(sv + i * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t x = (w[e] & EXP) ^ EXP;  // a field of zeros: infinity or NaN
              odd = odd || (F::WIDE ? !(x & 0xffffu) || !(x >> 16)
                                    : !(x & 0xffu) || !(x & 0xff00u) || !(x & 0xff0000u) || !(x >> 24));
            }
          }
          odd = __ballot(odd) != 0;
        }
        if (!odd) {
#pragma unroll
          for (int i = 0; i < DT; ++i) {
            bf16x8 vf;
            if constexpr (F::WIDE) {
              const int row = 4 * g + (col >> 2), in = 8 * (col & 1), c = 2 * i + ((col & 3) >> 1);
              const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(sv + row * ROW + v_chunk<CH, true>(row, c) * 16 + in));
              const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                  (lds_s16x4)(sv + (row + 16) * ROW + v_chunk<CH, true>(row + 16, c) * 16 + in));
              vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
            } else {
              const int j = col >> 1, row = 4 * g + (j & 3) + 4 * (j & 4);
              const i32x2 v = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                  (lds_i32x2)(sv + row * ROW + v_chunk<CH, false>(row, i) * 16 + 8 * (col & 1)));
              vf = codes8<FMT>((uint32_t)v[0], (uint32_t)v[1]);
            }
#pragma unroll
            for (int b = 0; b < RB; ++b) acc[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[b], acc[b][i], 0, 0, 0);
          }
        } else {
#pragma unroll 1
          for (int j = 0; j < SLICE; ++j) {  // a key at a time, for the rows that see it
            const int key = kb + j;
            float pj[RB];
#pragma unroll
            for (int b = 0; b < RB; ++b) {  // key j's probability lies in lane 16 (j / 4 % 4) + col, element 4 (j / 16) + j % 4
              float mine = 0.f;
#pragma unroll
              for (int e = 0; e < 8; ++e) mine = (j >> 4) * 4 + (j & 3) == e ? pr[b][e] : mine;
              pj[b] = __shfl(mine, ((j >> 2) & 3) * 16 + col, 64);
            }
#pragma unroll
            for (int i = 0; i < DT; ++i) {
              float v[4];  // dimensions 16 i + 4 g + r
              if constexpr (F::WIDE) {
                const int d = i * 16 + 4 * g;
                const uint2 w = *reinterpret_cast<const uint2*>(sv + j * ROW + v_chunk<CH, true>(j, d >> 3) * 16 + (d & 7) * 2);
                v[0] = bf16_bits_to_f32((uint16_t)w.x), v[1] = bf16_bits_to_f32((uint16_t)(w.x >> 16));
                v[2] = bf16_bits_to_f32((uint16_t)w.y), v[3] = bf16_bits_to_f32((uint16_t)(w.y >> 16));
              } else {
                const int w = *reinterpret_cast<const int*>(sv + j * ROW + v_chunk<CH, false>(j, i) * 16 + 4 * g);
                const auto v01 = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), v23 = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
                v[0] = v01[0], v[1] = v01[1], v[2] = v23[0], v[3] = v23[1];
              }
#pragma unroll
              for (int b = 0; b < RB; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[b][i][r] += key <= pos[b] && key >= lo[b] ? pj[b] * v[r] : 0.f;
              __builtin_amdgcn_sched_barrier(0);  // (one read at a time: this path must not cost the others registers)
            }
          }
        }
        lds_wait();
        if (t + NS < n) request_v(t + NS);
      };
      // Two loops, so that what masks need takes no registers from the slices without: they are nearly all of them
      const auto is_masked = [&](int t) { return key0 + t * UNIT + SLICE - 1 > min_pos || key0 + t * UNIT < max_lo; };
      for (int t = 0; t < n;) {
        for (; t < n && !is_masked(t); ++t) slice(t, std::false_type{});
        for (; t < n && is_masked(t); ++t) slice(t, std::true_type{});
      }
    }

    // ---- the waves' parts to LDS, where the slices were
#pragma unroll
    for (int b = 0; b < RB; ++b) l[b] = row_sum(l[b]);
    __syncthreads();
    float* so = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      if (g == 0) sml[wave * TR + b * 16 + col] = m[b], sml[(4 + wave) * TR + b * 16 + col] = l[b];
#pragma unroll
      for (int i = 0; i < DT; ++i)
        *reinterpret_cast<f32x4*>(so + ((wave * (DH / 4) + 4 * i + g) * TR + b * 16 + col) * 4) = acc[b][i];
    }
    __syncthreads();
    paged_finish<TR>(a, p, q, part, worker, so, sml);
    at += part.steps;
    if (at >= p.end) break;
    paged_next<TR>(a, p, q);
  }
}

constexpr int MT_ROWS = 128, MT_KEYS = 64;

template <int DH, int FMT>
struct Many {
  static constexpr bool WIDE = FMT == KEEP_CACHE_BF16;
  static constexpr int ROW = DH * 2, CH = ROW / 16;             // bytes and chunks of a key in LDS (bf16)
  static constexpr int TILE = MT_KEYS * ROW;                    // bytes of a tile of K or of V
  static constexpr int SC = 4 * TILE, TBL = SC + 2 * 2 * MT_KEYS * 4, LDS = TBL + TABLE * 4;
};

// Where a tile's 16-byte chunks lie: a K read is 32 rows at one chunk (16 at a time), a transposing V read four rows of four chunks.
template <int CH>
__device__ __forceinline__ int mk_chunk(int row, int c) {
  return CH == 16 ? c ^ (row & 15) : c ^ ((row >> 1) & 7);
}
template <int CH>
__device__ __forceinline__ int mv_chunk(int row, int c) {
  return CH == 16 ? c ^ (4 * (row & 3)) : c ^ (4 * ((row >> 1) & 1));
}

template <int DH, int FMT>
__global__ void __launch_bounds__(256, 2) k_paged_many(PagedArgs a) {
  using F = Many<DH, FMT>;
  constexpr int TR = MT_ROWS, KT = MT_KEYS, ROW = F::ROW, CH = F::CH, KS = DH / 16, NT = DH / 32;
  extern __shared__ __attribute__((aligned(256))) char lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, lq = lane & 31;
  const int worker = (blockIdx.x & 7) * (PAGED_WORKERS / 8) + (blockIdx.x >> 3);  // (neighbouring runs on one XCD)
  PagedSeq q;
  PagedPlace p = paged_place<TR, KT>(a, worker, reinterpret_cast<uint64_t*>(lds), q);
  if (tid == 0) a.rec[worker].last = 0;
  if (p.begin >= p.end) return;
  float* scales = reinterpret_cast<float*>(lds + F::SC);  // [2 buffers][64 of keys (with the scores' factor), 64 of values]
  int32_t* tbl = reinterpret_cast<int32_t*>(lds + F::TBL);
  const uint32_t lds_at = __builtin_amdgcn_readfirstlane(lds_address(lds));
  const int block_units = (int)max((int64_t)1, min((int64_t)1 << 20, (int64_t)(TABLE - 2) * a.c.page_size / KT));
  const float factor = fabsf(a.scale_log2e);

  // This lane's first operand chunks inside a tile: the others differ by one exclusive or, as the chunks' places do.  (Formed
  // anew in every tile: kept, they would push registers out to memory.)
  const int k_first = lq * ROW + mk_chunk<CH>(lq, g) * 16;
  int v_first;
  {
    const int vr = 4 * g + ((lane & 15) >> 2), c = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    v_first = vr * ROW + mv_chunk<CH>(vr, c) * 16 + 8 * (lane & 1);
  }

  for (uint64_t at = p.begin;;) {
    const PagedPart part = paged_part<TR, KT>(a, p, q, at);
    if (part.u0 == part.u1) break;  // (the run's last step)
    // ---- this lane's query row, and what the wave's rows see: keys up to pos, from lo on
    const int rows = q.rows * a.rep;
    int pos, lo;
    // the wave's last key and first one, and the keys that every row of the tile sees (lanes without a row are not stored)
    int max_pos = -1, min_lo = 0;
    const int min_pos = q.len - q.rows + (int)div_by(p.tile * TR, a.by_rep);
    const int max_lo = paged_from(q.len - q.rows + (int)div_by(min(rows, (p.tile + 1) * TR) - 1, a.by_rep), a.window);
    {
      const int x0 = p.tile * TR + wave * 32, x1 = min(rows, x0 + 32) - 1;
      if (x0 < rows) {
        max_pos = q.len - q.rows + (int)div_by(x1, a.by_rep);
        min_lo = paged_from(q.len - q.rows + (int)div_by(x0, a.by_rep), a.window);
      }
    }
    bf16x8 qf[KS];
    {
      const int x = p.tile * TR + wave * 32 + lq;
      const bool valid = x < rows;
      const int token = valid ? (int)div_by(x, a.by_rep) : 0, head = p.head * a.rep + (valid ? x - token * a.rep : 0);
      pos = valid ? q.len - q.rows + token : -1;
      lo = paged_from(pos, a.window);
      const __bf16* qp = static_cast<const __bf16*>(a.q) + (int64_t)(q.row0 + token) * a.q_stride + (int64_t)head * DH + g * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        u32x4 u = *reinterpret_cast<const u32x4*>(qp + ks * 16);
        if (F::WIDE && a.scale_log2e < 0.f) u ^= 0x80008000u;  // (the maximum is taken of products: their factor is positive)
        qf[ks] = __builtin_bit_cast(bf16x8, u);
      }
    }
    f32x16 acc[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[nt][e] = 0.f;
    float m = -INFINITY, l = 0.f;
    const int32_t* table = a.table + (int64_t)p.seq * a.max_pages;
    const int64_t head_at = (int64_t)p.head * a.c.head_stride;

    for (int ub = part.u0; ub < part.u1; ub += block_units) {
      const int ue = min(part.u1, ub + block_units), kt0 = part.first + ub, kt1 = part.first + ue;
      const int page0 = (int)div_by((uint32_t)kt0 * KT, a.by_page);
      const int page1 = (int)div_by((uint32_t)min((int64_t)kt1 * KT - 1, (int64_t)max(q.len, 1) - 1), a.by_page);
      __syncthreads();  // earlier entries, or the tiles of the job before, have been read
      for (int i = tid; i <= page1 - page0; i += 256) tbl[i] = min(max(table[page0 + i], 0), a.c.n_pages - 1);
      __syncthreads();
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));  // (in registers before the tiles' loads begin)

      // ---- tile kt to buffer `buf`.  bf16: straight to LDS.  8 bits: 16 codes of a row per load, kept in registers until the
      // other buffer has been used.  A wave loads 16 rows of a tile, RW per load with LPR lanes each.  Keys past the end read the
      // last one again and are masked.
      constexpr int LPR = DH * (F::WIDE ? 2 : 1) / 16, RW = 64 / LPR, NL = 16 / RW;
      const auto row_of = [&](int j) { return F::WIDE ? wave * 16 + j : j / RW * (4 * RW) + wave * RW + j % RW; };
      u32x4 kc[F::WIDE ? 1 : NL], vc[F::WIDE ? 1 : NL];
      float sc = 0.f;
      const int last = max(q.len, 1) - 1;
      const auto find = [&](int key, int& page, int& in) {
        const int n = (int)div_by(min(key, last), a.by_page);
        in = min(key, last) - n * a.c.page_size;
        page = tbl[n - page0];
      };
      // Where row lane % 16 of this wave's share of tile kt lies, in 16 bytes: formed a tile ahead of its loads
      const auto locate = [&](int kt) {
        int page, in, ln = lane;
        asm volatile("" : "+v"(ln));
        find(kt * KT + row_of(ln & 15), page, in);
        return (uint32_t)((page * a.c.page_stride + in * a.c.token_stride + head_at) * (F::WIDE ? 2 : 1) / 16);
      };
      const auto request = [&](int kt, int buf, uint32_t where) {
        int ln = lane;
        asm volatile("" : "+v"(ln));  // (what follows from the lane is formed anew: kept, it would push registers out to memory)
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          const int row = row_of(i * RW + ln / LPR);
          const int64_t e = (int64_t)(uint32_t)__shfl((int)where, i * RW + ln / LPR, 64) * 16;
          const char* k = static_cast<const char*>(a.c.k) + e;
          const char* v = static_cast<const char*>(a.c.v) + e;
          if constexpr (F::WIDE) {
            const uint32_t to = lds_at + buf * 2 * F::TILE + (wave * 16 + i * RW) * ROW;
            load_lds16(k + mk_chunk<CH>(row, ln % CH) * 16, to);
            load_lds16(v + mv_chunk<CH>(row, ln % CH) * 16, to + F::TILE);
          } else {
            kc[i] = *reinterpret_cast<const u32x4*>(k + (ln % LPR) * 16);
            vc[i] = *reinterpret_cast<const u32x4*>(v + (ln % LPR) * 16);
          }
        }
        if (!F::WIDE && tid < 2 * KT) {
          int page, in;
          find(kt * KT + (tid & (KT - 1)), page, in);
          const int64_t s = ((int64_t)page * a.c.n_kv_heads + p.head) * a.c.page_size + in;
          sc = tid < KT ? a.c.k_scale[s] * a.scale_log2e : a.c.v_scale[s];
        }
      };
      const auto arrive = [&](int buf) {
        if constexpr (F::WIDE) {
          vm_wait<0>();
        } else {
          char* to = lds + buf * 2 * F::TILE;
          int ln = lane;
          asm volatile("" : "+v"(ln));
#pragma unroll
          for (int i = 0; i < NL; ++i) {
            const int row = row_of(i * RW + ln / LPR), c = 2 * (ln % LPR);
            *reinterpret_cast<bf16x8*>(to + row * ROW + mk_chunk<CH>(row, c) * 16) = codes8<FMT>(kc[i][0], kc[i][1]);
            *reinterpret_cast<bf16x8*>(to + row * ROW + mk_chunk<CH>(row, c + 1) * 16) = codes8<FMT>(kc[i][2], kc[i][3]);
            *reinterpret_cast<bf16x8*>(to + F::TILE + row * ROW + mv_chunk<CH>(row, c) * 16) = codes8<FMT>(vc[i][0], vc[i][1]);
            *reinterpret_cast<bf16x8*>(to + F::TILE + row * ROW + mv_chunk<CH>(row, c + 1) * 16) = codes8<FMT>(vc[i][2], vc[i][3]);
          }
          if (tid < 2 * KT) scales[buf * 2 * KT + tid] = sc;
        }
      };

      request(kt0, 0, locate(kt0));
      uint32_t where = locate(min(kt0 + 1, kt1 - 1));
      arrive(0);
      __syncthreads();
      // One tile; MASKED: some row of the workgroup does not see some key of it
      const auto tile = [&](int kt, auto masked_type) __attribute__((always_inline)) {
        constexpr bool MASKED = decltype(masked_type)::value;
        const int cur = (kt - kt0) & 1, k0 = kt * KT;
        // every wave finished reading the other buffer before the barrier that ended the last iteration
        if (kt + 1 < kt1) {
          request(kt + 1, cur ^ 1, where);
          where = locate(min(kt + 2, kt1 - 1));
        }
        if (!MASKED || (k0 <= max_pos && k0 + KT > min_lo)) {
          const char* sk = lds + cur * 2 * F::TILE;
          const char* sv = sk + F::TILE;
          const float* ksc = scales + cur * 2 * KT;
          int k_at = k_first, v_at = v_first;
          asm volatile("" : "+v"(k_at), "+v"(v_at));
          // S^T for the two halves of the keys; K operands are read four steps ahead, the first V operands before the softmax (8
          // bits: the next tile's codes take the registers for that)
          f32x16 s[2];
          bf16x8 kf[2 * KS];
          const auto read_k = [&](int from) {
#pragma unroll
            for (int i = from; i < from + 4; ++i)
              if (i < 2 * KS) kf[i] = *reinterpret_cast<const bf16x8*>(sk + i / KS * 32 * ROW + (k_at ^ (i % KS * 32)));
          };
          s16x4 vf[2][NT][2];
          const auto read_v = [&](int step) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int b = 0; b < 2; ++b)
                vf[step & 1][nt][b] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(sv + (step * 16 + b * 8) * ROW + (v_at ^ (nt * 64))));
          };
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[h][e] = 0.f;
          read_k(0);
          read_k(4);
#pragma unroll
          for (int i = 0; i < 2 * KS; ++i) {
            s[i / KS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i], qf[i % KS], s[i / KS], 0, 0, 0);
            if (i % 4 == 3) read_k(i + 5);
            if (F::WIDE && i == 2 * KS - 5) read_v(0);
          }
          // ---- scores (8 bits: in the log2 domain already), mask, running maximum
          if constexpr (!F::WIDE) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const f32x4 f = *reinterpret_cast<const f32x4*>(ksc + h * 32 + 8 * i + 4 * g);
#pragma unroll
                for (int e = 0; e < 4; ++e) s[h][4 * i + e] *= f[e];
              }
          }
          if constexpr (MASKED) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const int key = k0 + h * 32 + 8 * (e >> 2) + 4 * g + (e & 3);
                s[h][e] = key <= pos && key >= lo ? s[h][e] : -INFINITY;
              }
          }
          float top = -INFINITY;
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s[h][e]);
          {
            auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            top = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
          }
          if (F::WIDE) top *= factor;
          const float m_new = fmaxf(m, top), ref = m_new == -INFINITY ? 0.f : m_new;
          if (__ballot(m_new != m)) {  // rescale only where some row's maximum moved
            const float alpha = __builtin_amdgcn_exp2f(m - ref);
            l *= alpha;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 16; ++e) acc[nt][e] *= alpha;
            m = m_new;
          }
          // fma(s, factor, -ref) keeps s factor exact, so the rounding of ref multiplies all of a row's weights alike and leaves
          // their quotients; from 2^31 on it would be all there is of them (2^128, or nothing).  Rows whose maximum lies beyond
          // FAR, where it could reach 2, round the products first, as it was.
          constexpr float FAR = 16777216.f;
          float by = factor;
          if (F::WIDE && __ballot(fabsf(ref) > FAR)) {
            const bool far = fabsf(ref) > FAR;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int e = 0; e < 16; ++e) s[h][e] = far ? s[h][e] * factor : s[h][e];
            by = far ? 1.f : factor;
          }
          uint32_t pk[2][8];
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
              float p0 = __builtin_amdgcn_exp2f(F::WIDE ? __builtin_fmaf(s[h][e], by, -ref) : s[h][e] - ref);
              float p1 = __builtin_amdgcn_exp2f(F::WIDE ? __builtin_fmaf(s[h][e + 1], by, -ref) : s[h][e + 1] - ref);
              l += p0 + p1;
              if constexpr (!F::WIDE) {
                const float* v = ksc + KT + h * 32 + 8 * (e >> 2) + 4 * g + (e & 3);
                p0 = MASKED && s[h][e] == -INFINITY ? 0.f : p0 * v[0];  // (a scale of NaN stays with the rows that see the key)
                p1 = MASKED && s[h][e + 1] == -INFINITY ? 0.f : p1 * v[1];
              }
              pk[h][e >> 1] = pack_bf16x2(p0, p1);
            }
          bool odd = false;
          if constexpr (MASKED && FMT != KEEP_CACHE_INT8) {
            // A product with a probability of zero would carry infinities and NaN to rows that do not see the key.
#pragma unroll 2
            for (int i = lane; i < F::TILE / 16; i += 64) {
              const u32x4 w = *reinterpret_cast<const u32x4*>(sv + i * 16);
#pragma unroll
              for (int e = 0; e < 4; ++e) odd = odd || (w[e] & 0x7f80u) == 0x7f80u || (w[e] & 0x7f800000u) == 0x7f800000u;
            }
            odd = __ballot(odd) != 0;
          }
          if (!odd) {
            // slot (g, i) of step s holds key 16 s + 8 (i / 4) + 4 g + i % 4: the keys of P^T's registers as they are
            if (!F::WIDE) read_v(0);
#pragma unroll
            for (int step = 0; step < 4; ++step) {
              if (step + 1 < 4) read_v(step + 1);
              u32x4 pu;
#pragma unroll
              for (int i = 0; i < 4; ++i) pu[i] = pk[step >> 1][(step & 1) * 4 + i];
              const bf16x8 pf = __builtin_bit_cast(bf16x8, pu);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
                acc[nt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    __builtin_bit_cast(bf16x8, __builtin_shufflevector(vf[step & 1][nt][0], vf[step & 1][nt][1], 0, 1, 2, 3, 4, 5, 6, 7)),
                    pf, acc[nt], 0, 0, 0);
            }
          } else {
#pragma unroll 1
            for (int j = 0; j < KT; ++j) {  // a key at a time, for the rows that see it
              uint32_t two = 0;  // key j lies in lane half (j / 4) % 2, element 4 (j % 32 / 8) + j % 4 of half-tile j / 32
              const int want = (j >> 5) * 8 + ((j & 31) >> 3) * 2 + ((j & 3) >> 1);
#pragma unroll
              for (int i = 0; i < 16; ++i) two = want == i ? pk[i >> 3][i & 7] : two;
              two = (uint32_t)__shfl((int)two, ((j >> 2) & 1) * 32 + lq, 64);
              const float pj = bf16_bits_to_f32((uint16_t)(j & 1 ? two >> 16 : two));
              const bool sees = k0 + j <= pos && k0 + j >= lo;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {  // dimensions 32 nt + 8 i + 4 g + r
                  const uint2 w = *reinterpret_cast<const uint2*>(sv + j * ROW + mv_chunk<CH>(j, 4 * nt + i) * 16 + 8 * g);
                  const uint32_t u[2] = {w.x, w.y};
#pragma unroll
                  for (int r = 0; r < 4; ++r)
                    acc[nt][4 * i + r] += sees ? pj * bf16_bits_to_f32((uint16_t)(u[r >> 1] >> (16 * (r & 1)))) : 0.f;
                  __builtin_amdgcn_sched_barrier(0);  // (one read at a time: this path must not cost the others registers)
                }
            }
          }
        }
        if (kt + 1 < kt1) arrive(cur ^ 1);
        __syncthreads();
      };
      // Two loops, so that what masks need takes no registers from the tiles without: they are nearly all of them
      const auto is_masked = [&](int kt) { return kt * KT + KT - 1 > min_pos || kt * KT < max_lo; };
      for (int kt = kt0; kt < kt1;) {
        for (; kt < kt1 && !is_masked(kt); ++kt) tile(kt, std::false_type{});
        for (; kt < kt1 && is_masked(kt); ++kt) tile(kt, std::true_type{});
      }
    }

    // ---- the job's result, or its part
    l += __shfl_xor(l, 32, 64);
    const bool whole = part.u0 == 0 && part.u1 == part.units;
    const int64_t slot = 2 * worker + (part.u0 == 0 ? 1 : 0);
    int x = wave * 32 + lq;
    asm volatile("" : "+v"(x));  // (the row's place is formed again here, not kept over the loop)
    x += p.tile * TR;
    const bool valid = x < rows;
    const int token = valid ? (int)div_by(x, a.by_rep) : 0, head = p.head * a.rep + (valid ? x - token * a.rep : 0);
    if (valid && whole) {
      const float inv = l != 0.f ? 1.f / l : 0.f;
      uint16_t* op = static_cast<uint16_t*>(a.out) + (int64_t)(q.row0 + token) * a.out_stride + (int64_t)head * DH;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          *reinterpret_cast<uint2*>(op + nt * 32 + 2 * e + 4 * g) =
              make_uint2(pack_bf16x2(acc[nt][e] * inv, acc[nt][e + 1] * inv), pack_bf16x2(acc[nt][e + 2] * inv, acc[nt][e + 3] * inv));
      if (g == 0 && a.lse) a.lse[(int64_t)(q.row0 + token) * a.n_q_heads + head] = 0.6931471805599453f * (m + log2f(l));
    } else if (valid) {
      const int row = wave * 32 + lq;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          *reinterpret_cast<f32x4*>(a.part_o + ((slot * (DH / 4) + ((nt * 32 + 2 * e + 4 * g) >> 2)) * TR + row) * 4) =
              f32x4{acc[nt][e], acc[nt][e + 1], acc[nt][e + 2], acc[nt][e + 3]};
      if (g == 0) {
        a.part_ml[slot * 2 * TR + row] = m;
        a.part_ml[(slot * 2 + 1) * TR + row] = l;
      }
    }
    if (tid == 0 && part.u0 == 0 && !whole)
      a.rec[worker] = PagedRecord{paged_worker_of(part.last, p.total), q.row0, p.tile * TR, min(TR, rows - p.tile * TR), p.head};
    at += part.steps;
    if (at >= p.end) break;
    paged_next<TR>(a, p, q);
  }
}

template <int DH>
void launch_many(const PagedArgs& a, hipStream_t s) {
  static std::atomic<uint64_t> done[3];
  const int f = a.c.format == KEEP_CACHE_BF16 ? 0 : a.c.format == KEEP_CACHE_FP8 ? 1 : 2;
  const auto kernel = f == 0 ? k_paged_many<DH, KEEP_CACHE_BF16> : f == 1 ? k_paged_many<DH, KEEP_CACHE_FP8> : k_paged_many<DH, KEEP_CACHE_INT8>;
  constexpr int bytes = Many<DH, KEEP_CACHE_BF16>::LDS;
  set_max_dyn_smem_once(done[f], reinterpret_cast<const void*>(kernel), bytes);
  hipLaunchKernelGGL(kernel, dim3(PAGED_WORKERS), dim3(256), (size_t)bytes, s, a);
}

template <int DH, int FMT, int RB>
void launch_few(const PagedArgs& a, hipStream_t s) {
  static std::atomic<uint64_t> done{0};
  const auto kernel = k_paged_few<DH, FMT, RB>;
  set_max_dyn_smem_once(done, reinterpret_cast<const void*>(kernel), Few<DH, FMT, RB>::LDS);
  hipLaunchKernelGGL(kernel, dim3(PAGED_WORKERS), dim3(256), (size_t)(Few<DH, FMT, RB>::LDS), s, a);
}
template <int DH, int RB>
void launch_few_format(const PagedArgs& a, hipStream_t s) {
  if (a.c.format == KEEP_CACHE_BF16)
    launch_few<DH, KEEP_CACHE_BF16, RB>(a, s);
  else if (a.c.format == KEEP_CACHE_FP8)
    launch_few<DH, KEEP_CACHE_FP8, RB>(a, s);
  else
    launch_few<DH, KEEP_CACHE_INT8, RB>(a, s);
}

}  // namespace

void launch_paged_mfma(const PagedArgs& a, int rows, hipStream_t s) {
  if (a.c.head_dim == 256)
    rows == 16 ? launch_few_format<256, 1>(a, s) : launch_few<256, KEEP_CACHE_BF16, 2>(a, s);
  else if (rows == MT_ROWS)
    a.c.head_dim == 128 ? launch_many<128>(a, s) : launch_many<64>(a, s);
  else if (a.c.head_dim == 128)
    rows == 16 ? launch_few_format<128, 1>(a, s) : launch_few_format<128, 2>(a, s);
  else
    rows == 16 ? launch_few_format<64, 1>(a, s) : launch_few_format<64, 2>(a, s);
  launch_paged_join(a, rows, s);
}

}  // namespace keep
