// What the kernels of paged attention share: arguments, the division of a launch's work, partial results.
//
// Work.  A job is (sequence, key/value head, tile of TR query rows); a query row is a token paired with one of the head's query
// heads.  A job takes as many units as it has key tiles of KT keys between the first key its rows may see and the
// last, at least one (so that rows which see nothing are written too).  The work of a launch, in the order sequence, head,
// tile, key, is dealt to the workers (workgroups) in equal runs: lengths differ by orders of magnitude from
// sequence to sequence, and their division has to come from device memory, where a captured graph finds the
// step's own.  Every worker forms the division for itself: sums per sequence in LDS, a scan, then its own place.
// Beginning a job takes about as long as a unit (tables, queries, the first loads, the output), so a job weighs one step more than
// its units, the first of them without keys.
//
// A job cut by a border between runs leaves one partial result per worker: unnormalised output, running maximum and sum.  A
// worker cuts at most the job it begins with (slot 2 w) and the one it ends with (slot 2 w + 1); the worker a cut job begins in
// leaves a record, by which k_paged_join adds the parts in the order of their keys.
#pragma once
#include "serve_common.h"

namespace keep {

constexpr int PAGED_WORKERS = 512;  // two workgroups for each of 256 CUs

struct PagedRecord {  // of a worker: the cut job that begins in it
  int32_t last;       // the last worker of that job; 0: no such job
  int32_t row0;       // first query row of the sequence
  int32_t x0, n;      // the tile's query rows: the first (within sequence and head) and their number
  int32_t head;
};

struct PagedArgs {
  keep_paged_cache c;
  const void* q;
  void* out;
  float* lse;
  const int32_t *q_start, *kv_len, *table;
  int64_t q_stride, out_stride;
  int n_seqs, n_rows, n_q_heads, rep, max_pages, window, capacity, dtype;
  float scale_log2e;
  FastDiv by_page, by_rep;
  PagedRecord* rec;  // [PAGED_WORKERS]
  float* part_ml;    // [2 PAGED_WORKERS][2][TR]: maximum (log2 domain), sum
  float* part_o;     // [2 PAGED_WORKERS][head_dim / 4][TR][4]
};

struct PagedSeq {
  int row0, rows, len;  // first query row, their number, tokens in the cache
};

__device__ __forceinline__ PagedSeq paged_seq(const PagedArgs& a, int s) {
  PagedSeq q;
  q.row0 = min(max(a.q_start[s], 0), a.n_rows);
  q.rows = min(max(a.q_start[s + 1], q.row0), a.n_rows) - q.row0;
  q.len = min(max(a.kv_len[s], 0), a.capacity);
  return q;
}

// The same number in every lane, kept in a scalar register so that what depends on it branches and loads as one
__device__ __forceinline__ int paged_uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ uint64_t paged_uniform(uint64_t v) {
  return (uint64_t)(uint32_t)paged_uniform((int)(v >> 32)) << 32 | (uint32_t)paged_uniform((int)v);
}
__device__ __forceinline__ PagedSeq paged_uniform(PagedSeq q) {
  return PagedSeq{paged_uniform(q.row0), paged_uniform(q.rows), paged_uniform(q.len)};
}

// First key that a row at position pos sees.  A row before the first token counts as the first one, so that no window, however
// long, takes the difference below -2^31.
__host__ __device__ __forceinline__ int paged_from(int pos, int window) {
  const int from = (pos < 0 ? 0 : pos) - window + 1;
  return window == 0 || from < 0 ? 0 : from;
}

// Key tiles of one tile of query rows: [first, first + units)
template <int TR, int KT>
__host__ __device__ __forceinline__ void paged_span(const PagedArgs& a, const PagedSeq& q, int tile, int& first, int& units) {
  const int rows = q.rows * a.rep, end = (tile + 1) * TR, x1 = rows < end ? rows : end;
  const int last = q.len - q.rows + (int)div_by(x1 - 1, a.by_rep);
  const int from = q.len - q.rows + (int)div_by(tile * TR, a.by_rep);
  first = paged_from(from, a.window) / KT;
  units = last < 0 ? 1 : last / KT + 1 - first;
  if (last < 0) first = 0;
}
template <int TR>
__host__ __device__ __forceinline__ int paged_tiles(const PagedArgs& a, const PagedSeq& q) {
  return (q.rows * a.rep + TR - 1) / TR;
}

// Every worker that takes part has a step at least
__device__ __forceinline__ uint64_t paged_workers(uint64_t total) { return min(total, (uint64_t)PAGED_WORKERS); }
// The worker that takes step v: the largest w with w * total / workers <= v
__device__ __forceinline__ int paged_worker_of(uint64_t v, uint64_t total) {
  return (int)(((v + 1) * paged_workers(total) - 1) / total);
}

struct PagedPlace {    // where a worker begins, and how far it goes
  uint64_t total;      // steps of the launch
  uint64_t begin, end; // this worker's run
  int seq, head, tile;
  int step;            // steps of the first job that earlier workers take
};

// Called by all 256 threads; lds: 8 * (n_seqs + 260) bytes, free again after the caller's next barrier.  q: the sequence the
// worker begins with.
template <int TR, int KT>
__device__ __forceinline__ PagedPlace paged_place(const PagedArgs& a, int worker, uint64_t* lds, PagedSeq& q) {
  const int tid = threadIdx.x;
  uint64_t* sums = lds + 260;
  for (int s = tid; s < a.n_seqs; s += 256) sums[s] = 0;
  __syncthreads();
  // a few sequences: several threads add up the tiles of one; many: a thread takes every 256th
  int share = 1;
  while (share * 2 * a.n_seqs <= 256) share *= 2;
  for (int s = tid / share; s < a.n_seqs; s += 256 / share) {
    const PagedSeq one = paged_seq(a, s);
    const int tiles = paged_tiles<TR>(a, one);
    uint64_t sum = 0;
    for (int t = tid & (share - 1); t < tiles; t += share) {
      int first, units;
      paged_span<TR, KT>(a, one, t, first, units);
      sum += units + 1;
    }
    if (sum) atomicAdd(reinterpret_cast<unsigned long long*>(sums + s), (unsigned long long)sum);
  }
  __syncthreads();
  const int per = (a.n_seqs + 255) / 256;
  const int s0 = min(tid * per, a.n_seqs), s1 = min(s0 + per, a.n_seqs);
  uint64_t own = 0;
  for (int s = s0; s < s1; ++s) own += sums[s];
  uint64_t before = own;  // inclusive scan over the wave, then over the waves
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t up = __shfl_up((unsigned long long)before, o, 64);
    if ((tid & 63) >= o) before += up;
  }
  if ((tid & 63) == 63) lds[tid >> 6] = before;
  __syncthreads();
  uint64_t total = 0;
  for (int w = 0; w < 4; ++w) {
    if (w < (tid >> 6)) before += lds[w];
    total += lds[w];
  }
  before = (before - own) * a.c.n_kv_heads;
  own *= a.c.n_kv_heads;
  PagedPlace p{};
  p.total = paged_uniform(total * a.c.n_kv_heads);
  static_assert((PAGED_WORKERS & (PAGED_WORKERS - 1)) == 0, "the runs are found by shifts");
  const bool many = p.total >= PAGED_WORKERS;
  p.begin = many ? p.total * worker / PAGED_WORKERS : min((uint64_t)worker, p.total);
  p.end = many ? p.total * (worker + 1) / PAGED_WORKERS : min((uint64_t)worker + 1, p.total);
  if (p.begin >= p.end) return p;
  if (p.begin >= before && p.begin < before + own) {  // one thread
    int s = s0, head = 0;
    uint64_t at = p.begin - before;
    while (at >= sums[s] * a.c.n_kv_heads) at -= sums[s++] * a.c.n_kv_heads;
    while (at >= sums[s]) at -= sums[s], ++head;
    lds[8] = (uint64_t)(uint32_t)head << 32 | (uint32_t)s;
    lds[9] = at;
  }
  __syncthreads();
  p.seq = paged_uniform((int)lds[8]);
  p.head = paged_uniform((int)(lds[8] >> 32));
  uint64_t at = paged_uniform(lds[9]);
  // the tile: 64 at a time, a lane each
  q = paged_uniform(paged_seq(a, p.seq));
  const int tiles = paged_tiles<TR>(a, q), lane = tid & 63;
  for (int t0 = 0; t0 < tiles; t0 += 64) {
    int first, units = -1;
    if (t0 + lane < tiles) paged_span<TR, KT>(a, q, t0 + lane, first, units);
    uint64_t sum = units + 1;
    for (int o = 1; o < 64; o <<= 1) {
      const uint64_t up = __shfl_up((unsigned long long)sum, o, 64);
      if (lane >= o) sum += up;
    }
    const uint64_t past = __ballot(sum > at);
    if (past) {
      const int l = __ffsll((unsigned long long)past) - 1;
      p.tile = t0 + l;
      p.step = paged_uniform((int)(at - (l ? __shfl((unsigned long long)sum, l - 1, 64) : 0)));
      break;
    }
    at -= paged_uniform((uint64_t)__shfl((unsigned long long)sum, 63, 64));
  }
  return p;
}

// The part of a job that a worker takes: units [u0, u1), none where it has the first step alone
struct PagedPart {
  int first, units, u0, u1;  // units: of the whole job; first: key tile of unit 0
  int steps;                 // steps of the worker's run that it uses up
  uint64_t last;             // the job's last step
};
template <int TR, int KT>
__device__ __forceinline__ PagedPart paged_part(const PagedArgs& a, const PagedPlace& p, const PagedSeq& q, uint64_t at) {
  PagedPart r;
  paged_span<TR, KT>(a, q, p.tile, r.first, r.units);
  const int c1 = (int)min((uint64_t)r.units + 1, p.step + (p.end - at));
  r.u0 = max(p.step - 1, 0);
  r.u1 = c1 - 1;
  r.steps = c1 - p.step;
  r.last = at - p.step + r.units;
  return r;
}

// The job behind (seq, head, tile); sequences without rows are passed over.  Only called where another job exists.
template <int TR>
__device__ __forceinline__ void paged_next(const PagedArgs& a, PagedPlace& p, PagedSeq& q) {
  p.step = 0;
  if (++p.tile < paged_tiles<TR>(a, q)) return;
  p.tile = 0;
  if (++p.head < a.c.n_kv_heads) return;
  p.head = 0;
  do q = paged_uniform(paged_seq(a, ++p.seq));
  while (q.rows == 0 && p.seq + 1 < a.n_seqs);
}

typedef __attribute__((ext_vector_type(4))) float paged_f32x4;

// The four waves' parts of a job (each of other keys), added in their order: the job's result, or a partial one where the job
// was cut.  so: LDS [4 waves][head_dim / 4][TR][4]; sml: LDS [2][4 waves][TR], maxima and sums.
template <int TR>
__device__ __forceinline__ void paged_finish(const PagedArgs& a, const PagedPlace& p, const PagedSeq& q, const PagedPart& part,
                                             int worker, const float* so, const float* sml) {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));  // (what follows from it is formed here, not kept in registers from job to job)
  const int row = tid % TR, quads = a.c.head_dim / 4;
  const int x = p.tile * TR + row;
  const bool valid = x < q.rows * a.rep, whole = part.u0 == 0 && part.u1 == part.units;
  const int token = valid ? (int)div_by(x, a.by_rep) : 0, head = p.head * a.rep + (valid ? x - token * a.rep : 0);
  const int64_t slot = 2 * worker + (part.u0 == 0 ? 1 : 0);
  float mw[4], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) m = fmaxf(m, mw[w] = sml[w * TR + row]);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    mw[w] = mw[w] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw[w] - m);
    l += sml[(4 + w) * TR + row] * mw[w];
  }
  for (int d4 = tid / TR; d4 < quads; d4 += 256 / TR) {
    paged_f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const paged_f32x4 v = *reinterpret_cast<const paged_f32x4*>(so + ((w * quads + d4) * TR + row) * 4);
      o += mw[w] == 0.f ? paged_f32x4{0.f, 0.f, 0.f, 0.f} : v * mw[w];
    }
    if (!valid) continue;
    if (!whole) {
      *reinterpret_cast<paged_f32x4*>(a.part_o + ((slot * quads + d4) * TR + row) * 4) = o;
    } else {
      if (l != 0.f) o /= l;
      const int64_t o_at = (int64_t)(q.row0 + token) * a.out_stride + (int64_t)head * a.c.head_dim + d4 * 4;
      if (a.dtype == KEEP_F32)
        *reinterpret_cast<paged_f32x4*>(static_cast<float*>(a.out) + o_at) = o;
      else
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + o_at) =
            make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
    }
  }
  if (tid < TR) {
    if (!whole) {
      a.part_ml[slot * 2 * TR + row] = m;
      a.part_ml[(slot * 2 + 1) * TR + row] = l;
    } else if (valid && a.lse) {
      a.lse[(int64_t)(q.row0 + token) * a.n_q_heads + head] = 0.6931471805599453f * (m + log2f(l));
    }
  }
  if (tid == 0 && part.u0 == 0 && !whole)
    a.rec[worker] = PagedRecord{paged_worker_of(part.last, p.total), q.row0, p.tile * TR, min(TR, q.rows * a.rep - p.tile * TR),
                                p.head};
}

void launch_paged_generic(const PagedArgs& a, int rows, hipStream_t s);  // tiles of 16 or 32 query rows
// bf16 queries, heads of 64, 128 or 256, a bf16 or 8-bit cache of less than 64 GB per tensor; rows: query rows of a tile (16, 32 or
// 128; heads of 256 16, with bf16 keys 32 too)
void launch_paged_mfma(const PagedArgs& a, int rows, hipStream_t s);
void launch_paged_join(const PagedArgs& a, int rows, hipStream_t s);

}  // namespace keep
