// Sampling one token per row from given uniform numbers: temperature, min-p, top-k, top-p.
//
// Tokens weigh w_i = rint(2^40 exp(-(X - x_i) / T)), whole numbers, and are ranked by logit and then by id.  Every limit keeps a
// prefix of that ranking, and the choice itself is the first prefix that outweighs a goal, so all that is ever asked is: which
// token in rank brings the number of tokens (or their weight) to a goal?  No sort of the row is needed for that:
//   1. the largest logit X;
//   2. a histogram of the tokens over t = log2(e) (X - x) / T, which rises with the rank: their number per bin, and their weight
//      but where top_k bounds their number (light: no weight is formed yet); min_p bounds t;
//   3. the tokens of the bins in which the goals can lie are listed: light all bins up to the limit, else a bin or two per goal;
//   4. the list is sorted and summed, and the goals are found in it.
// Sums are of whole numbers, so neither atomics nor the division among threads can change a result.  A row is read three times
// (HBM the first time).  A list that does not fit (thousands of equal or nearly equal logits in a bin) is left to find_token,
// which divides the bin further by the bits of the logits.  Few rows are divided among workgroups, a launch per step, with the
// histogram and the list in the workspace; else a workgroup does a whole row in LDS.
#include <algorithm>

#include "serve_common.h"

namespace keep {
namespace {

constexpr int ST = 512;               // threads of a row's workgroup (1024 would leave each 128 registers: spills)
constexpr int BINS = 2048;
constexpr double T_MAX = 41.25;       // beyond t = 41 a weight rounds to zero
constexpr double T_SCALE = BINS / T_MAX;
constexpr double ONE = 1099511627776.0;  // 2^40
constexpr int LIST = 2048;            // tokens that are ranked among themselves
constexpr int MAX_PARTS = 16;
// Rows are divided up to 64 of them, and from 40 000 tokens on: a launch per step costs some 15 us more than one kernel.  us divided /
// whole: 64 rows of 16 000 29 / 17, 32 000 30 / 20 (weighing all 43 / 37), 64 000 30 / 27, 152 064 weighing all 67 / 110;
// 128 rows of 152 064 57 / 49.
constexpr int WIDE_ROWS = 64, WIDE_VOCAB = 40000;

// Larger numbers first, NaN last; -0 equals +0
__device__ __forceinline__ uint32_t order_key(float v) {
  if (v != v) return 0;
  const uint32_t u = v == 0.f ? 0u : __float_as_uint(v);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ uint64_t token_key(float v, int id) { return (uint64_t)order_key(v) << 32 | ~(uint32_t)id; }

// The same number in every lane, kept in scalar registers
__device__ __forceinline__ uint64_t uniform64(uint64_t v) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v);
}

struct Row {
  const void* x;
  int dtype, n;
  bool vec;            // 16-byte pieces
  float top;           // X
  double c;            // log2(e) / temperature
  double t_cut;        // tokens beyond it are out: min_p, or a weight of zero
  uint64_t w_min;
  __device__ float at(int i) const {
    return dtype == KEEP_F32 ? static_cast<const float*>(x)[i] : bf16_bits_to_f32(static_cast<const uint16_t*>(x)[i]);
  }
  __device__ double place(float v) const { return v == top ? 0.0 : ((double)top - (double)v) * c; }  // t, NaN for NaN
  // no token with t <= limit lies below it
  __device__ float floor_of(double limit) const {
    const double span = limit / c, f = (double)top - span - 1e-6 * (fabs((double)top) + span);
    return f > -3e38 && f < 3e38 ? (float)f : -INFINITY;  // (an infinite X, an infinite temperature: all)
  }
  __device__ int bin(double t) const { return min(BINS - 1, (int)(t * T_SCALE)); }
  // rint(2^(40 - t)), t = k + f: the series of 2^-f = exp(-f ln 2) to its twelfth power (|f| <= 1/2: 2e-16 is left out).  Adding
  // 2^52 rounds to a whole number and leaves it in the low bits.
  __device__ uint64_t weight(double t) const {
    if (!(t < T_MAX)) return 0;
    const double k = rint(t), z = (t - k) * -0.6931471805599453;
    double p = fma(z, 1.0 / 479001600, 1.0 / 39916800);
    p = fma(z, p, 1.0 / 3628800);
    p = fma(z, p, 1.0 / 362880);
    p = fma(z, p, 1.0 / 40320);
    p = fma(z, p, 1.0 / 5040);
    p = fma(z, p, 1.0 / 720);
    p = fma(z, p, 1.0 / 120);
    p = fma(z, p, 1.0 / 24);
    p = fma(z, p, 1.0 / 6);
    p = fma(z, p, 0.5);
    p = fma(z, p, 1.0);
    p = fma(z, p, 1.0);
    return __double_as_longlong(ldexp(p, 40 - (int)k) + 4503599627370496.0) & 0xfffffffffffffull;
  }
  __device__ uint64_t stays(double t) const {  // the weight, zero below min_p
    const uint64_t w = t <= t_cut ? weight(t) : 0;
    return w >= w_min ? w : 0;
  }
};

// piece(first id, logits[N]) for the tokens [begin, end) of a row (begin a multiple of 8) in 16-byte pieces, eight loads of a thread
// at a time, then one(id, logit) for those behind the last whole piece, or for all where the row is not aligned
template <int N, typename P, typename O>
__device__ __forceinline__ void each_piece(const Row& r, int begin, int end, P piece, O one) {
  int whole = begin;
  if (r.vec) {
    whole = begin + (end - begin) / N * N;
    for (int i = begin + (int)threadIdx.x * N; i < whole; i += 8 * ST * N) {
      uint4 u[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)  // (a piece past the end reads the last one again)
        u[j] = *reinterpret_cast<const uint4*>(static_cast<const char*>(r.x) + (int64_t)min(i + j * ST * N, whole - N) * (16 / N));
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t w[4] = {u[j].x, u[j].y, u[j].z, u[j].w};
        float v[N];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (N == 4) {
            v[e] = __uint_as_float(w[e]);
          } else {
            v[2 * e] = bf16_bits_to_f32((uint16_t)w[e]);
            v[2 * e + 1] = bf16_bits_to_f32((uint16_t)(w[e] >> 16));
          }
        }
        if (i + j * ST * N < whole) piece(i + j * ST * N, v);
      }
    }
  }
  for (int i = whole + (int)threadIdx.x; i < end; i += ST) one(i, r.at(i));
}

// f(id, logit) for the tokens [begin, end) whose logit is at least `floor` (most pieces hold none: one comparison)
template <typename F>
__device__ __forceinline__ void each_token(const Row& r, int begin, int end, float floor, F f) {
  const auto one = [&](int i, float v) {
    if (v >= floor) f(i, v);
  };
  const auto piece = [&](int i, const auto& v) {
    constexpr int N = sizeof(v) / sizeof(v[0]);
    float top = v[0];
#pragma unroll
    for (int e = 1; e < N; ++e) top = fmaxf(top, v[e]);
    if (!(top >= floor)) return;
#pragma unroll
    for (int e = 0; e < N; ++e) one(i + e, v[e]);
  };
  if (r.dtype == KEEP_F32)
    each_piece<4>(r, begin, end, piece, one);
  else
    each_piece<8>(r, begin, end, piece, one);
}

struct Found {
  uint64_t upto;  // weights up to and with the token
  uint64_t w;
  int id;
};

// Bins whose tokens are listed, in up to three stretches.  Of a token in stretch j the weight (number) ranked before it is what
// the list holds before it and add_mass (add_count).
struct Plan {
  int mode;                  // below
  int n;                     // stretches; the others hold no bin
  int first[3], last[3];
  uint64_t add_mass[3];
  uint32_t add_count[3];
  uint64_t total;            // weight of all that min_p leaves; 0: not known (light)
  uint32_t listed;           // tokens of the stretches
};
enum { PLAN_LIST = 0, PLAN_WEIGH = 1, PLAN_FIND = 2 };  // go on / light did not fit / neither did

struct ListLds {
  uint64_t key[LIST];
  uint32_t rank[256];
  uint64_t wave_sum[16], stays;
};

struct SampleLds {
  uint64_t mass[BINS];   // inclusive sums along the bins
  uint32_t count[BINS];
  union {
    ListLds sort;
    struct {
      uint64_t w[LIST];
      float x[LIST];
      int id[LIST];
    } list;
    struct {
      uint64_t mass[BINS];
      uint32_t count[BINS];
    } digit;
  };
  uint64_t wave_mass[ST / 64];
  uint32_t wave_count[ST / 64];
  uint64_t bin_mass;     // of the bin found: weight and number before it
  uint32_t bin_count, bin_n;
  int bin, listed;
  uint64_t stays;
  Found found;
  Plan plan;
};

// Inclusive sums of two histograms of BINS entries, neighbours per thread
__device__ __forceinline__ void scan_bins(uint64_t* mass, uint32_t* count, SampleLds& l) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  constexpr int PER = BINS / ST;
  uint64_t m = 0;
  uint32_t c = 0;
#pragma unroll
  for (int e = 0; e < PER; ++e) m += mass[PER * t + e], c += count[PER * t + e];
  const uint64_t own_m = m;
  const uint32_t own_c = c;
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t um = __shfl_up((unsigned long long)m, o, 64);
    const uint32_t uc = __shfl_up(c, o, 64);
    if (lane >= o) m += um, c += uc;
  }
  if (lane == 63) l.wave_mass[wave] = m, l.wave_count[wave] = c;
  __syncthreads();
  for (int w = 0; w < wave; ++w) m += l.wave_mass[w], c += l.wave_count[w];
  m -= own_m, c -= own_c;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    m += mass[PER * t + e], c += count[PER * t + e];
    mass[PER * t + e] = m, count[PER * t + e] = c;
  }
  __syncthreads();
}

// The bin in which the inclusive sums reach `goal`
__device__ __forceinline__ void find_bin(const uint64_t* mass, const uint32_t* count, uint64_t goal, bool by_mass, SampleLds& l) {
  for (int b = threadIdx.x; b < BINS; b += ST) {
    const uint64_t m0 = b ? mass[b - 1] : 0;
    const uint32_t c0 = b ? count[b - 1] : 0;
    if (by_mass ? m0 < goal && goal <= mass[b] : c0 < goal && goal <= count[b]) {
      l.bin = b;
      l.bin_mass = m0;
      l.bin_count = c0;
      l.bin_n = count[b] - c0;
    }
  }
  __syncthreads();
}

// The token in rank that brings the number of tokens, or their weight, to `goal` (1 .. what there is)
__device__ __forceinline__ Found find_token(const Row& r, uint64_t goal, bool by_mass, SampleLds& l) {
  find_bin(l.mass, l.count, goal, by_mass, l);
  const int bin = __builtin_amdgcn_readfirstlane(l.bin);
  uint64_t before = uniform64(l.bin_mass);
  uint32_t n = __builtin_amdgcn_readfirstlane(l.bin_n);
  goal = uniform64(goal - (by_mass ? l.bin_mass : l.bin_count));
  uint32_t prefix = 0;  // leading bits of the logits' order that are settled
  int shift = 32;
  const auto in_bin = [&](int i, float& v, uint64_t& w) {
    v = r.at(i);
    const double t = r.place(v);
    if (!(t <= r.t_cut) || r.bin(t) != bin) return false;
    w = r.stays(t);
    return w != 0 && (shift == 32 || order_key(v) >> shift == prefix);
  };
  while (n > LIST && shift > 0) {
    const int bits = shift == 32 ? 11 : shift == 21 ? 11 : 10;
    __syncthreads();
    for (int b = threadIdx.x; b < BINS; b += ST) l.digit.mass[b] = 0, l.digit.count[b] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < r.n; i += ST) {
      float v;
      uint64_t w;
      if (!in_bin(i, v, w)) continue;
      const int b = (1 << bits) - 1 - (int)(order_key(v) >> (shift - bits) & ((1u << bits) - 1));  // larger logits first
      atomicAdd(reinterpret_cast<unsigned long long*>(l.digit.mass + b), (unsigned long long)w);
      atomicAdd(l.digit.count + b, 1u);
    }
    __syncthreads();
    scan_bins(l.digit.mass, l.digit.count, l);
    find_bin(l.digit.mass, l.digit.count, goal, by_mass, l);
    before = uniform64(before + l.bin_mass);
    goal = uniform64(goal - (by_mass ? l.bin_mass : l.bin_count));
    n = __builtin_amdgcn_readfirstlane(l.bin_n);
    prefix = (prefix << bits) | ((1u << bits) - 1 - (uint32_t)__builtin_amdgcn_readfirstlane(l.bin));
    shift -= bits;
  }
  __syncthreads();
  if (n > LIST) {
    // equal logits, and many: the goal's place among them is a division, its id the place's in id order
    const uint64_t w = r.stays(r.place(key_value(prefix)));
    const uint32_t place = (uint32_t)(by_mass ? (goal - 1) / w : goal - 1);
    uint32_t seen = 0;
    for (int i0 = 0; i0 < r.n; i0 += ST) {
      const int i = i0 + threadIdx.x;
      const bool is = i < r.n && order_key(r.at(i)) == prefix;
      const uint64_t waves = __ballot(is);
      if ((threadIdx.x & 63) == 0) l.wave_count[threadIdx.x >> 6] = __popcll(waves);
      __syncthreads();
      uint32_t mine = seen, all = seen;
      for (int v = 0; v < ST / 64; ++v) {
        if (v < (int)(threadIdx.x >> 6)) mine += l.wave_count[v];
        all += l.wave_count[v];
      }
      mine += __popcll(waves & ((1ull << (threadIdx.x & 63)) - 1));
      if (is && mine == place) l.found = Found{before + (place + 1) * w, w, i};
      seen = all;
      __syncthreads();
      if (seen > place) break;
    }
    return l.found;
  }
  if (threadIdx.x == 0) l.listed = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < r.n; i += ST) {
    float v;
    uint64_t w;
    if (!in_bin(i, v, w)) continue;
    const int at = atomicAdd(&l.listed, 1);
    l.list.w[at] = w;
    l.list.x[at] = v;
    l.list.id[at] = i;
  }
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < n; e += ST) {
    const float v = l.list.x[e];
    const int id = l.list.id[e];
    uint64_t mass = 0;
    uint32_t count = 0;
    for (uint32_t f = 0; f < n; ++f) {
      const bool first = l.list.x[f] > v || (l.list.x[f] == v && l.list.id[f] < id);
      mass += first ? l.list.w[f] : 0;
      count += first;
    }
    const uint64_t w = l.list.w[e];
    if (by_mass ? mass < goal && goal <= mass + w : count + 1 == goal) l.found = Found{before + mass + w, w, id};
  }
  __syncthreads();
  return l.found;
}

struct SampleArgs {
  const void* logits;
  int64_t row_stride;
  int dtype, n_rows, vocab;
  const float *uniform, *temperature;  // NULL: the values below
  const int32_t* top_k;
  const float *top_p, *min_p;
  float temperature0, top_p0, min_p0;
  int32_t top_k0;
  int32_t none;  // token of a row without a number
  int32_t* tokens;
  float* probs;
  // few rows: a row's tokens in parts of part_len (a multiple of 8), and in the workspace
  int parts, part_len;
  uint64_t* best;      // [rows][MAX_PARTS] largest token_key of each part
  uint64_t* mass;      // [rows][BINS]
  uint32_t* count;     // [rows][BINS]
  uint64_t* list;      // [rows][LIST] token_keys
  Plan* plan;          // [rows]
  int32_t* listed;     // [rows]
};

// ---- the steps; every thread of the workgroup takes part in each -------------------------------------------------
__device__ __forceinline__ Row row_of(const SampleArgs& a, int row) {
  Row r{};
  r.x = static_cast<const char*>(a.logits) + (int64_t)row * a.row_stride * (a.dtype == KEEP_F32 ? 4 : 2);
  r.dtype = a.dtype;
  r.n = a.vocab;
  r.vec = (reinterpret_cast<uintptr_t>(r.x) & 15) == 0;
  return r;
}

// Of the tokens [begin, end) the largest token_key
__device__ __forceinline__ uint64_t largest(const Row& r, int begin, int end, SampleLds& l) {
  float top = -INFINITY;
  int id = -1;
  // (a thread meets rising ids: an equal logit does not replace.  NaN loses every comparison)
  const auto one = [&](int i, float v) {
    if (v > top) top = v, id = i;
  };
  int at = -1;  // the piece with the thread's largest logit
  const auto piece = [&](int i, const auto& v) {
    constexpr int N = sizeof(v) / sizeof(v[0]);
    float t = v[0];
#pragma unroll
    for (int e = 1; e < N; ++e) t = fmaxf(t, v[e]);
    if (t > top) top = t, at = i;
  };
  if (r.dtype == KEEP_F32)
    each_piece<4>(r, begin, end, piece, [](int, float) {});
  else
    each_piece<8>(r, begin, end, piece, [](int, float) {});
  if (at >= 0) {
    id = at;
    while (r.at(id) != top) ++id;
  }
  const int per = r.dtype == KEEP_F32 ? 4 : 8, whole = r.vec ? begin + (end - begin) / per * per : begin;
  for (int i = whole + (int)threadIdx.x; i < end; i += ST) one(i, r.at(i));
  uint64_t best = id < 0 ? 0 : token_key(top, id);
  for (int o = 32; o > 0; o >>= 1) {
    const uint64_t other = __shfl_xor((unsigned long long)best, o, 64);
    best = other > best ? other : best;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) l.wave_mass[threadIdx.x >> 6] = best;
  __syncthreads();
  for (int w = 0; w < ST / 64; ++w) best = l.wave_mass[w] > best ? l.wave_mass[w] : best;
  __syncthreads();
  return best;
}

// What the row asks for.  The five numbers are fetched by five lanes at once: one after the other they would cost a launch of
// few rows their latency each.
struct Wishes {
  float temperature, top_p, min_p, u;
  int32_t k;
  bool light;
};
__device__ __forceinline__ Wishes wishes_of(const SampleArgs& a, int row) {
  const int lane = threadIdx.x & 63;
  const void* from = lane == 0 ? a.temperature : lane == 1 ? (const void*)a.top_k : lane == 2 ? a.top_p : lane == 3 ? a.min_p : a.uniform;
  uint32_t bits = lane == 1 ? (uint32_t)a.top_k0 : __float_as_uint(lane == 0 ? a.temperature0 : lane == 2 ? a.top_p0 : a.min_p0);
  if (lane < 5 && from) bits = static_cast<const uint32_t*>(from)[row];
  Wishes w;
  w.temperature = __uint_as_float(__builtin_amdgcn_readlane(bits, 0));
  w.k = (int32_t)__builtin_amdgcn_readlane(bits, 1);
  w.top_p = __uint_as_float(__builtin_amdgcn_readlane(bits, 2));
  w.min_p = __uint_as_float(__builtin_amdgcn_readlane(bits, 3));
  const float u = __uint_as_float(__builtin_amdgcn_readlane(bits, 4));
  if (w.k < 1) w.k = INT32_MAX;
  if (!(w.top_p < 1.f)) w.top_p = 1.f;  // (and NaN)
  w.u = u >= 0.f ? fminf(u, 1.f - 1.f / 16777216.f) : 0.f;
  w.light = w.k <= LIST / 2;
  return w;
}

// The scale of a row with this largest token; false where the choice is made already (thread 0 writes it if `write`)
__device__ __forceinline__ bool set_scale(const SampleArgs& a, int row, uint64_t best, bool write, const Wishes& w, Row& r) {
  best = uniform64(best);
  const uint32_t key = (uint32_t)(best >> 32);
  r.top = key_value(key);
  if (key <= 0x007fffffu || !(w.temperature > 0.f)) {  // nothing above -infinity, or greedy
    if (write && threadIdx.x == 0) {
      const bool none = key <= 0x007fffffu;
      a.tokens[row] = none ? a.none : (int32_t)~(uint32_t)best;
      if (a.probs) a.probs[row] = none ? 0.f : 1.f;
    }
    return false;
  }
  r.c = 1.4426950408889634 / (double)w.temperature;
  r.w_min = 1;
  r.t_cut = T_MAX;
  if (w.min_p > 0.f) {
    r.w_min = max((uint64_t)1, (uint64_t)ceil(fmin((double)w.min_p, 1.0) * ONE));
    // (a binary32 logarithm is good to 1e-5 here: tokens below min_p by less are weighed and found too light)
    r.t_cut = fmin(T_MAX, -log2f(fminf(w.min_p, 1.f)) + 1e-4);
  }
  r.c = __longlong_as_double(uniform64(__double_as_longlong(r.c)));
  r.t_cut = __longlong_as_double(uniform64(__double_as_longlong(r.t_cut)));
  r.w_min = uniform64(r.w_min);
  return true;
}

__device__ __forceinline__ void clear_bins(SampleLds& l) {
  for (int b = threadIdx.x; b < BINS; b += ST) l.mass[b] = 0, l.count[b] = 0;
  __syncthreads();
}

// Number of the tokens [begin, end) per bin, and their weight unless LIGHT (then those below min_p by a hair are counted too)
template <bool LIGHT>
__device__ __forceinline__ void histogram(const Row& r, int begin, int end, SampleLds& l) {
  each_token(r, begin, end, r.floor_of(r.t_cut), [&](int, float v) {
    const double t = r.place(v);
    if (!(t <= r.t_cut)) return;
    const int b = r.bin(t);
    if constexpr (!LIGHT) {
      const uint64_t w = r.stays(t);
      if (w == 0) return;
      atomicAdd(reinterpret_cast<unsigned long long*>(l.mass + b), (unsigned long long)w);
    }
    atomicAdd(l.count + b, 1u);
  });
  __syncthreads();
}

// The weight at which top_p cuts, of `mass` in all
__device__ __forceinline__ uint64_t share_of(double top_p, uint64_t mass) {
  if (top_p >= 1.0) return mass;
  const double share = ceil(top_p * (double)mass);
  return share >= 1.0 ? min((uint64_t)share, mass) : 1;
}
__device__ __forceinline__ uint64_t goal_of(double u, uint64_t mass) { return min((uint64_t)floor(u * (double)mass), mass - 1) + 1; }

// From the scanned histogram the bins to list (into l.plan, by all threads together)
__device__ __forceinline__ void make_plan(const Row& r, const Wishes& w, bool light, SampleLds& l) {
  const uint32_t all = l.count[BINS - 1];
  const bool limited = (uint32_t)w.k < all;
  int first[3], last[3];  // of the choice, of top_p's end, of top_k's end; none: first > last
  for (int i = 0; i < 3; ++i) first[i] = BINS, last[i] = -1;
  if (light) {
    first[0] = 0, last[0] = BINS - 1;
    if (limited) {
      find_bin(l.mass, l.count, w.k, false, l);
      last[0] = l.bin;
    }
  } else {
    // weight of what top_k leaves: between lo and hi, as far as the bin of its last token tells
    const auto bin_at = [&](uint64_t goal) {
      __syncthreads();
      find_bin(l.mass, l.count, goal, true, l);
      return __builtin_amdgcn_readfirstlane(l.bin);
    };
    uint64_t lo = uniform64(l.mass[BINS - 1]), hi = lo;
    if (limited) {
      find_bin(l.mass, l.count, w.k, false, l);
      first[2] = last[2] = l.bin;
      lo = l.bin_mass + 1, hi = l.mass[l.bin];
    }
    if (w.top_p < 1.0) {
      first[1] = bin_at(share_of(w.top_p, lo)), last[1] = bin_at(share_of(w.top_p, hi));
      lo = min(lo, first[1] ? l.mass[first[1] - 1] + 1 : 1), hi = min(hi, l.mass[last[1]]);
    }
    first[0] = bin_at(goal_of(w.u, lo)), last[0] = bin_at(goal_of(w.u, hi));
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    // the stretches in rising order, those that touch made one
    Plan& p = l.plan;
    p.n = 0;
    p.total = light || limited ? 0 : l.mass[BINS - 1];
    uint64_t mass = 0;
    uint32_t count = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      if (first[i] > last[i]) continue;
      const int end = p.n ? p.last[p.n - 1] : -2;
      if (first[i] <= end + 1) {
        if (last[i] <= end) continue;
        mass += l.mass[last[i]] - l.mass[end];
        count += l.count[last[i]] - l.count[end];
        p.last[p.n - 1] = last[i];
        continue;
      }
      const uint64_t m0 = first[i] ? l.mass[first[i] - 1] : 0;
      const uint32_t c0 = first[i] ? l.count[first[i] - 1] : 0;
      p.first[p.n] = first[i], p.last[p.n] = last[i];
      p.add_mass[p.n] = m0 - mass, p.add_count[p.n] = c0 - count;
      ++p.n;
      mass += l.mass[last[i]] - m0;
      count += l.count[last[i]] - c0;
    }
    for (int i = p.n; i < 3; ++i) p.first[i] = BINS, p.last[i] = -1, p.add_mass[i] = 0, p.add_count[i] = 0;
    p.listed = count;
    p.mode = count <= LIST ? PLAN_LIST : light ? PLAN_WEIGH : PLAN_FIND;
  }
  __syncthreads();
}

__device__ __forceinline__ int stretch_of(const Plan& p, int bin) {
  return bin >= p.first[0] && bin <= p.last[0] ? 0 : bin >= p.first[1] && bin <= p.last[1] ? 1
         : bin >= p.first[2] && bin <= p.last[2] ? 2 : -1;
}

// put(token_key) for the tokens [begin, end) of the plan's bins
template <typename F>
__device__ __forceinline__ void list_tokens(const Row& r, const Plan& p, int begin, int end, bool light, F put) {
  const int a0 = p.first[0], b0 = p.last[0], a1 = p.first[1], b1 = p.last[1], a2 = p.first[2], b2 = p.last[2];
  const double far = fmin(r.t_cut, (max(b0, max(b1, b2)) + 1.001) / T_SCALE);  // (nearly all tokens lie beyond the last bin)
  each_token(r, begin, end, r.floor_of(far), [&](int i, float v) {
    const double t = r.place(v);
    if (!(t <= far)) return;
    const int b = r.bin(t);
    if (((b >= a0 && b <= b0) || (b >= a1 && b <= b1) || (b >= a2 && b <= b2)) && (light || r.stays(t))) put(token_key(v, i));
  });
}

// The list in l.key, n of it, sorted and summed by NT threads: the goals in it.  PER neighbours per thread.
template <int NT>
__device__ __forceinline__ void choose(const SampleArgs& a, int row, const Row& r, const Wishes& w, const Plan& plan, int n, ListLds& l) {
  constexpr int PER = LIST / NT;
  const int tid = threadIdx.x;
  if (tid == 0) l.stays = 0;
  if (n <= 256) {
    // few: every token's rank is the number of larger keys, counted by NT / size threads
    int size = 2;
    while (size < n) size *= 2;
    if (tid < size) l.rank[tid] = 0;
    __syncthreads();
    const int e = tid & (size - 1), step = NT / size;
    const uint64_t mine = e < n ? l.key[e] : 0;
    uint32_t larger = 0;
#pragma unroll 8
    for (int i = tid / size; i < n; i += step) larger += l.key[i] > mine;
    if (e < n && larger) atomicAdd(l.rank + e, larger);
    __syncthreads();
    if (tid < n) l.key[l.rank[tid]] = mine;
    __syncthreads();
  } else {
    int size = 512;
    while (size < n) size *= 2;
    for (int i = n + tid; i < size; i += NT) l.key[i] = 0;
    __syncthreads();
    for (int span = 2; span <= size; span *= 2)
      for (int half = span / 2; half > 0; half /= 2) {
        for (int t = tid; t < size / 2; t += NT) {
          const int i = 2 * t - (t & (half - 1)), j = i + half;
          const uint64_t x = l.key[i], y = l.key[j];
          if ((x < y) == ((i & span) == 0)) l.key[i] = y, l.key[j] = x;  // larger keys first
        }
        __syncthreads();
      }
  }
  // weights, their sums, what is ranked before
  uint64_t key[PER], weight[PER], after[PER], sum = 0;
  int stretch[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const int i = PER * tid + e;
    key[e] = weight[e] = 0, stretch[e] = 0;
    if (i < n) {
      key[e] = l.key[i];
      const double t = r.place(key_value((uint32_t)(key[e] >> 32)));
      weight[e] = r.weight(t);
      stretch[e] = max(0, stretch_of(plan, r.bin(t)));
    }
    sum += weight[e];
  }
  uint64_t upto = sum;
  if ((tid >> 6) * 64 * PER < n)
    for (int o = 1; o < 64; o <<= 1) {
      const uint64_t up = __shfl_up((unsigned long long)upto, o, 64);
      if ((tid & 63) >= o) upto += up;
    }
  if ((tid & 63) == 63) l.wave_sum[tid >> 6] = upto;
  __syncthreads();
  for (int v = 0; v < tid >> 6 && v * 64 * PER < n; ++v) upto += l.wave_sum[v];
#pragma unroll
  for (int e = PER - 1; e >= 0; --e) {
    after[e] = upto + plan.add_mass[stretch[e]];
    upto -= weight[e];
  }
  // what min_p and top_k leave ends with a token of the list, or is all there is
  uint64_t last = 0;
#pragma unroll
  for (int e = 0; e < PER; ++e)
    if (weight[e] >= r.w_min && (uint32_t)(PER * tid + e) + plan.add_count[stretch[e]] < (uint32_t)w.k) last = after[e];
  if (last) atomicMax(reinterpret_cast<unsigned long long*>(&l.stays), (unsigned long long)last);
  __syncthreads();
  uint64_t stays = plan.total ? plan.total : l.stays;
  const uint64_t share = share_of(w.top_p, stays);
  __syncthreads();
  if (share < stays) {
#pragma unroll
    for (int e = 0; e < PER; ++e)
      if (weight[e] != 0 && after[e] - weight[e] < share && share <= after[e]) l.stays = after[e];
    __syncthreads();
    stays = l.stays;
  }
  const uint64_t goal = goal_of(w.u, stays);
#pragma unroll
  for (int e = 0; e < PER; ++e)
    if (weight[e] != 0 && after[e] - weight[e] < goal && goal <= after[e]) {
      a.tokens[row] = (int32_t)~(uint32_t)key[e];
      if (a.probs) a.probs[row] = (float)((double)weight[e] / (double)stays);
    }
}

// The same from the scanned histogram with weights, by find_token: any number of tokens in any bin
__device__ __forceinline__ void choose_by_finding(const SampleArgs& a, int row, const Row& r, const Wishes& w, SampleLds& l) {
  uint64_t stays = uniform64(l.mass[BINS - 1]);
  const bool limited = (uint32_t)w.k < l.count[BINS - 1];
#pragma unroll 1
  for (int step = limited ? 0 : 1; step < 3; ++step) {  // the ends of top_k and top_p, the choice
    const uint64_t goal = step == 0 ? w.k : step == 1 ? share_of(w.top_p, stays) : goal_of(w.u, stays);
    if (step == 1 && goal >= stays) continue;
    __syncthreads();
    const Found f = find_token(r, goal, step > 0, l);
    if (step < 2) {
      stays = uniform64(f.upto);
    } else if (threadIdx.x == 0) {
      a.tokens[row] = f.id;
      if (a.probs) a.probs[row] = (float)((double)f.w / (double)stays);
    }
  }
}

// Steps 2 to 4 by one workgroup, from a histogram with weights on where the light one did not do
__device__ __forceinline__ void whole_row(const SampleArgs& a, int row, const Row& r, const Wishes& w, bool light, SampleLds& l) {
  if (light) {
    clear_bins(l);
    histogram<true>(r, 0, r.n, l);
    scan_bins(l.mass, l.count, l);
    make_plan(r, w, true, l);
    light = l.plan.mode == PLAN_LIST;
  }
  if (!light) {
    clear_bins(l);
    histogram<false>(r, 0, r.n, l);
    scan_bins(l.mass, l.count, l);
    make_plan(r, w, false, l);
    if (l.plan.mode == PLAN_FIND) return choose_by_finding(a, row, r, w, l);
  }
  if (threadIdx.x == 0) l.listed = 0;
  __syncthreads();
  list_tokens(r, l.plan, 0, r.n, light, [&](uint64_t key) {
    const int at = atomicAdd(&l.listed, 1);
    if (at < LIST) l.sort.key[at] = key;  // (always, as the histogram has counted them)
  });
  __syncthreads();
  choose<ST>(a, row, r, w, l.plan, min(LIST, l.listed), l.sort);
}

__global__ void __launch_bounds__(ST) k_sample_row(SampleArgs a) {
  __shared__ SampleLds l;
  const int row = blockIdx.x;
  Row r = row_of(a, row);
  const Wishes w = wishes_of(a, row);
  if (!set_scale(a, row, largest(r, 0, r.n, l), true, w, r)) return;
  whole_row(a, row, r, w, w.light, l);
}

// ---- few rows: blockIdx.x = part, blockIdx.y = row
__device__ __forceinline__ uint64_t best_of(const SampleArgs& a, int row) {
  static_assert(MAX_PARTS == 16, "a lane per part");
  const int p = threadIdx.x & 15;
  uint64_t best = p < a.parts ? a.best[(int64_t)row * MAX_PARTS + p] : 0;
  for (int o = 1; o < 16; o <<= 1) {
    const uint64_t other = __shfl_xor((unsigned long long)best, o, 64);
    best = other > best ? other : best;
  }
  return best;
}

__global__ void __launch_bounds__(ST) k_sample_max(SampleArgs a) {
  __shared__ SampleLds l;
  const int row = blockIdx.y, begin = blockIdx.x * a.part_len;
  const Row r = row_of(a, row);
  // (the next step's sums start from zero)
  for (int b = blockIdx.x * ST + threadIdx.x; b < BINS; b += gridDim.x * ST)
    a.mass[(int64_t)row * BINS + b] = 0, a.count[(int64_t)row * BINS + b] = 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) a.listed[row] = 0;
  const uint64_t best = largest(r, begin, min(r.n, begin + a.part_len), l);
  if (threadIdx.x == 0) a.best[(int64_t)row * MAX_PARTS + blockIdx.x] = best;
}

__global__ void __launch_bounds__(ST) k_sample_bins(SampleArgs a) {
  __shared__ SampleLds l;
  const int row = blockIdx.y, begin = blockIdx.x * a.part_len;
  Row r = row_of(a, row);
  const Wishes w = wishes_of(a, row);
  if (!set_scale(a, row, best_of(a, row), false, w, r)) return;
  clear_bins(l);
  if (w.light)
    histogram<true>(r, begin, min(r.n, begin + a.part_len), l);
  else
    histogram<false>(r, begin, min(r.n, begin + a.part_len), l);
  for (int b = threadIdx.x; b < BINS; b += ST)
    if (l.count[b]) {
      atomicAdd(a.count + (int64_t)row * BINS + b, l.count[b]);
      if (!w.light) atomicAdd(reinterpret_cast<unsigned long long*>(a.mass + (int64_t)row * BINS + b), (unsigned long long)l.mass[b]);
    }
}

__global__ void __launch_bounds__(ST) k_sample_list(SampleArgs a) {
  __shared__ SampleLds l;
  const int row = blockIdx.y, begin = blockIdx.x * a.part_len;
  Row r = row_of(a, row);
  const Wishes w = wishes_of(a, row);
  if (!set_scale(a, row, best_of(a, row), blockIdx.x == 0, w, r)) return;
  for (int b = threadIdx.x; b < BINS; b += ST) {
    l.mass[b] = a.mass[(int64_t)row * BINS + b];
    l.count[b] = a.count[(int64_t)row * BINS + b];
  }
  __syncthreads();
  scan_bins(l.mass, l.count, l);
  make_plan(r, w, w.light, l);
  if (blockIdx.x == 0 && threadIdx.x == 0) a.plan[row] = l.plan;
  if (l.plan.mode != PLAN_LIST) {  // (rare: one workgroup does the row)
    __syncthreads();
    if (blockIdx.x == 0) whole_row(a, row, r, w, false, l);
    return;
  }
  list_tokens(r, l.plan, begin, min(r.n, begin + a.part_len), w.light,
              [&](uint64_t key) {
                const int at = atomicAdd(a.listed + row, 1);
                if (at < LIST) a.list[(int64_t)row * LIST + at] = key;  // (always, as the histogram has counted them)
              });
}

constexpr int CT = 256;
__global__ void __launch_bounds__(CT) k_sample_choose(SampleArgs a) {
  __shared__ ListLds l;
  __shared__ Plan plan;
  __shared__ int listed;
  const int row = blockIdx.x;
  Row r{};
  // (everything that a row's choice reads is requested at once)
  const Wishes w = wishes_of(a, row);
  const uint64_t best = best_of(a, row);
  constexpr int WORDS = sizeof(Plan) / 4;
  static_assert(sizeof(Plan) % 4 == 0 && WORDS < CT, "a thread per word");
  if (threadIdx.x < WORDS) reinterpret_cast<uint32_t*>(&plan)[threadIdx.x] = reinterpret_cast<const uint32_t*>(a.plan + row)[threadIdx.x];
  if (threadIdx.x == WORDS) listed = a.listed[row];
#pragma unroll
  for (int i = 0; i < LIST / CT; ++i) l.key[i * CT + threadIdx.x] = a.list[(int64_t)row * LIST + i * CT + threadIdx.x];
  if (!set_scale(a, row, best, false, w, r)) return;  // (the step before has written the choice)
  __syncthreads();
  if (plan.mode == PLAN_LIST) choose<CT>(a, row, r, w, plan, min(LIST, listed), l);
}

// Bytes of the workspace's pieces for one row
constexpr int64_t ROW_BYTES = MAX_PARTS * 8 + BINS * 12 + LIST * 8 + sizeof(Plan) + 4;
bool is_wide(int32_t n_rows, int32_t vocab) { return n_rows <= WIDE_ROWS && vocab >= WIDE_VOCAB; }
uint64_t workspace_bytes(int32_t n_rows, int32_t vocab) {
  return is_wide(n_rows, vocab) ? 256 + n_rows * ((ROW_BYTES + 255) / 256 * 256) : 256;
}

void launch(SampleArgs a, void* workspace, hipStream_t s) {
  if (!is_wide(a.n_rows, a.vocab)) {
    hipLaunchKernelGGL(k_sample_row, dim3(a.n_rows), dim3(ST), 0, s, a);
    return;
  }
  // parts: 256 workgroups in all, 4096 tokens or more each
  a.parts = std::max(1, std::min({MAX_PARTS, 256 / a.n_rows, a.vocab / 4096}));
  a.part_len = ((a.vocab + a.parts - 1) / a.parts + 7) / 8 * 8;
  const int64_t n = a.n_rows;
  char* at = static_cast<char*>(workspace);
  const auto take = [&](int64_t bytes) {
    char* p = at;
    at += bytes;
    return p;
  };
  a.best = reinterpret_cast<uint64_t*>(take(n * MAX_PARTS * 8));
  a.mass = reinterpret_cast<uint64_t*>(take(n * BINS * 8));
  a.list = reinterpret_cast<uint64_t*>(take(n * LIST * 8));
  a.plan = reinterpret_cast<Plan*>(take(n * sizeof(Plan)));
  a.count = reinterpret_cast<uint32_t*>(take(n * BINS * 4));
  a.listed = reinterpret_cast<int32_t*>(take(n * 4));
  const dim3 grid(a.parts, a.n_rows);
  hipLaunchKernelGGL(k_sample_max, grid, dim3(ST), 0, s, a);
  hipLaunchKernelGGL(k_sample_bins, grid, dim3(ST), 0, s, a);
  hipLaunchKernelGGL(k_sample_list, grid, dim3(ST), 0, s, a);
  hipLaunchKernelGGL(k_sample_choose, dim3(a.n_rows), dim3(CT), 0, s, a);
}

}  // namespace

uint64_t sample_decode_bytes() { return workspace_bytes(1, KEEP_SAMPLE_MAX_VOCAB); }

void launch_sample_decode(const float* logits, int32_t vocab, const float* d_uniform, const keep_sampling& how, int32_t* token,
                          float* prob, void* workspace, hipStream_t s) {
  SampleArgs a{};
  a.logits = logits;
  a.row_stride = vocab;
  a.dtype = KEEP_F32;
  a.n_rows = 1;
  a.vocab = vocab;
  a.uniform = d_uniform;
  a.temperature0 = how.temperature;
  a.top_k0 = how.top_k;
  a.top_p0 = how.top_p;
  a.min_p0 = how.min_p;
  a.none = 0;
  a.tokens = token;
  a.probs = prob;
  launch(a, workspace, s);
}

}  // namespace keep

using namespace keep;

extern "C" uint64_t keep_sample_workspace_bytes(int32_t n_rows, int32_t vocab) {
  if (n_rows < 0 || n_rows > 65535 || vocab < 1 || vocab > KEEP_SAMPLE_MAX_VOCAB) return 0;
  return workspace_bytes(n_rows, vocab);
}

extern "C" keep_status keep_sample(const keep_sample_desc* d, const void* logits, const float* uniform,
                                   const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                                   int32_t* tokens, float* probs, void* workspace, uint64_t workspace_bytes, void* stream) {
  const char* me = "keep_sample";
  if (!d) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: desc is NULL", me);
  if (!is_dtype(d->dtype)) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: unknown dtype %d", me, d->dtype);
  if (d->n_rows < 0 || d->n_rows > 65535) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: n_rows %d outside [0, 65535]", me, d->n_rows);
  if (d->vocab < 1) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: vocab must be at least 1", me);
  if (d->vocab > KEEP_SAMPLE_MAX_VOCAB)
    return serve_fail(KEEP_ERR_SHAPE, "%s: vocab %d is above %d", me, d->vocab, KEEP_SAMPLE_MAX_VOCAB);
  if (d->row_stride < d->vocab) return serve_fail(KEEP_ERR_INVALID_ARG, "%s: row_stride is below vocab", me);
  if (d->n_rows == 0) return KEEP_OK;
  if (!logits || !uniform || !tokens || !workspace)
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: logits / uniform / tokens / workspace is NULL", me);
  if (reinterpret_cast<uintptr_t>(logits) % dtype_size(d->dtype) || reinterpret_cast<uintptr_t>(workspace) % 256)
    return serve_fail(KEEP_ERR_INVALID_ARG, "%s: logits or workspace is not aligned", me);
  if (workspace_bytes < keep_sample_workspace_bytes(d->n_rows, d->vocab))
    return serve_fail(KEEP_ERR_WORKSPACE, "%s: workspace of %llu bytes is too small", me, (unsigned long long)workspace_bytes);
  SampleArgs a{};
  a.logits = logits;
  a.row_stride = d->row_stride;
  a.dtype = d->dtype;
  a.n_rows = d->n_rows;
  a.vocab = d->vocab;
  a.uniform = uniform;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.temperature0 = a.top_p0 = 1.f;
  a.none = -1;
  a.tokens = tokens;
  a.probs = probs;
  launch(a, workspace, static_cast<hipStream_t>(stream));
  return launched(me);
}
