// Sampling one token per row from given uniform numbers: temperature, min-p, top-k, top-p.
//
// Tokens weigh w_i = rint(2^40 exp(-(X - x_i) / T)), whole numbers, and are ranked by logit and then by id.  Every limit keeps a
// prefix of that ranking, and the choice itself is the first prefix that outweighs a goal, so all that is ever asked is: which
// token in rank brings the number of tokens (or their weight) to a goal?  No sort is needed for that.  A histogram over
// y = (X - x) / T, which rises with the rank, finds the bin; the bin's few tokens are gathered and ranked among
// themselves; where they are many (equal or nearly equal logits) the bits of the logits divide the bin further.  Sums
// are of whole numbers, so neither atomics nor the division among threads can change a result.
#include <algorithm>

#include "serve_common.h"

namespace keep {
namespace {

constexpr int ST = 1024;              // threads of a row's workgroup
constexpr int BINS = 2 * ST;
constexpr double Y_MAX = 28.5;        // beyond y = 41 ln 2 = 28.42 a weight rounds to zero
constexpr double Y_SCALE = BINS / Y_MAX;
constexpr double ONE = 1099511627776.0;  // 2^40
constexpr int LIST = 2048;            // tokens that are ranked among themselves

// Larger numbers first, NaN last; -0 equals +0
__device__ __forceinline__ uint32_t order_key(float v) {
  if (v != v) return 0;
  const uint32_t u = v == 0.f ? 0u : __float_as_uint(v);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

struct Row {
  const void* x;
  int dtype, n;
  float top;      // X
  double t;       // temperature > 0
  uint64_t w_min; // lighter tokens are out (min_p)
  __device__ float at(int i) const {
    return dtype == KEEP_F32 ? static_cast<const float*>(x)[i] : bf16_bits_to_f32(static_cast<const uint16_t*>(x)[i]);
  }
  __device__ uint64_t weight(float v, int& bin) const {
    const double y = v == top ? 0.0 : ((double)top - (double)v) / t;
    if (!(y < Y_MAX)) return 0;  // (NaN too)
    bin = min(BINS - 1, (int)(y * Y_SCALE));
    const uint64_t w = (uint64_t)rint(exp(-y) * ONE);
    return w >= w_min ? w : 0;
  }
};

struct Found {
  uint64_t upto;  // weights up to and with the token
  uint64_t w;
  int id;
};

struct SampleLds {
  uint64_t mass[BINS];   // inclusive sums along the bins
  uint32_t count[BINS];
  union {
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
  Found found;
};

// Inclusive sums of two histograms of BINS entries, two entries per thread
__device__ __forceinline__ void scan_bins(uint64_t* mass, uint32_t* count, SampleLds& l) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const uint64_t m0 = mass[2 * t], m1 = mass[2 * t + 1];
  const uint32_t c0 = count[2 * t], c1 = count[2 * t + 1];
  uint64_t m = m0 + m1;
  uint32_t c = c0 + c1;
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t um = __shfl_up((unsigned long long)m, o, 64);
    const uint32_t uc = __shfl_up(c, o, 64);
    if (lane >= o) m += um, c += uc;
  }
  if (lane == 63) l.wave_mass[wave] = m, l.wave_count[wave] = c;
  __syncthreads();
  for (int w = 0; w < wave; ++w) m += l.wave_mass[w], c += l.wave_count[w];
  mass[2 * t] = m - m1, mass[2 * t + 1] = m;
  count[2 * t] = c - c1, count[2 * t + 1] = c;
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
__device__ Found find_token(const Row& r, uint64_t goal, bool by_mass, SampleLds& l) {
  find_bin(l.mass, l.count, goal, by_mass, l);
  const int bin = l.bin;
  uint64_t before = l.bin_mass;
  uint32_t n = l.bin_n;
  goal -= by_mass ? l.bin_mass : l.bin_count;
  // logits that may lie in the bin: a little more than it spans
  const double slack = 1e-9 * (fabs((double)r.top) + 30.0 * r.t);
  const double hi = (double)r.top - r.t * (bin / Y_SCALE) + slack, lo = (double)r.top - r.t * ((bin + 1) / Y_SCALE) - slack;
  // (an infinite X makes these NaN: then nothing is passed over)
  uint32_t prefix = 0;  // leading bits of the logits' order that are settled
  int shift = 32;
  const auto in_bin = [&](int i, float& v, uint64_t& w) {
    v = r.at(i);
    const double d = v;
    if (d < lo || d > hi) return false;
    int b = -1;
    w = r.weight(v, b);
    return w != 0 && b == bin && (shift == 32 || order_key(v) >> shift == prefix);
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
    before += l.bin_mass;
    goal -= by_mass ? l.bin_mass : l.bin_count;
    n = l.bin_n;
    prefix = (prefix << bits) | ((1u << bits) - 1 - (uint32_t)l.bin);
    shift -= bits;
  }
  __syncthreads();
  if (n > LIST) {
    // equal logits, and many: the goal's place among them is a division, its id the place's in id order
    int b;
    const uint64_t w = r.weight(key_value(prefix), b);
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
};

__global__ void __launch_bounds__(ST) k_sample_row(SampleArgs a) {
  __shared__ SampleLds l;
  __shared__ uint64_t wave_best[ST / 64];
  const int row = blockIdx.x, tid = threadIdx.x;
  Row r;
  r.x = static_cast<const char*>(a.logits) + (int64_t)row * a.row_stride * (a.dtype == KEEP_F32 ? 4 : 2);
  r.dtype = a.dtype;
  r.n = a.vocab;
  // ---- the largest logit, the lowest id among equals
  uint64_t best = 0;
  for (int i = tid; i < r.n; i += ST) {
    const uint64_t k = (uint64_t)order_key(r.at(i)) << 32 | ~(uint32_t)i;
    best = k > best ? k : best;
  }
  for (int o = 32; o > 0; o >>= 1) {
    const uint64_t other = __shfl_xor((unsigned long long)best, o, 64);
    best = other > best ? other : best;
  }
  if ((tid & 63) == 0) wave_best[tid >> 6] = best;
  for (int b = tid; b < BINS; b += ST) l.mass[b] = 0, l.count[b] = 0;
  __syncthreads();
  for (int w = 0; w < ST / 64; ++w) best = wave_best[w] > best ? wave_best[w] : best;
  const uint32_t best_key = (uint32_t)(best >> 32);
  r.top = key_value(best_key);
  r.t = a.temperature ? a.temperature[row] : a.temperature0;
  if (best_key <= 0x007fffffu || !(r.t > 0.0)) {  // nothing above -infinity, or greedy
    if (tid == 0) {
      const bool none = best_key <= 0x007fffffu;
      a.tokens[row] = none ? a.none : (int32_t)~(uint32_t)best;
      if (a.probs) a.probs[row] = none ? 0.f : 1.f;
    }
    return;
  }
  const double min_p = a.min_p ? a.min_p[row] : a.min_p0;
  r.w_min = min_p > 0.0 ? max((uint64_t)1, (uint64_t)ceil(fmin(min_p, 1.0) * ONE)) : 1;
  // ---- number and weight of the tokens per bin
  for (int i = tid; i < r.n; i += ST) {
    int b;
    const uint64_t w = r.weight(r.at(i), b);
    if (w == 0) continue;
    atomicAdd(reinterpret_cast<unsigned long long*>(l.mass + b), (unsigned long long)w);
    atomicAdd(l.count + b, 1u);
  }
  __syncthreads();
  scan_bins(l.mass, l.count, l);
  uint64_t stays = l.mass[BINS - 1];
  const int32_t k = a.top_k ? a.top_k[row] : a.top_k0;
  if (k >= 1 && (uint32_t)k < l.count[BINS - 1]) stays = find_token(r, k, false, l).upto;
  const double top_p = a.top_p ? a.top_p[row] : a.top_p0;
  if (top_p == top_p) {
    const double share = ceil(top_p * (double)stays);
    const uint64_t goal = share >= 1.0 ? (share < 18446744073709551615.0 ? (uint64_t)share : ~(uint64_t)0) : 1;
    __syncthreads();
    if (goal < stays) stays = find_token(r, goal, true, l).upto;
  }
  const float u0 = a.uniform[row];
  const double u = u0 >= 0.f ? fmin((double)u0, 1.0 - 1.0 / 16777216.0) : 0.0;
  const uint64_t goal = min((uint64_t)floor(u * (double)stays), stays - 1) + 1;
  __syncthreads();
  const Found f = find_token(r, goal, true, l);
  if (tid == 0) {
    a.tokens[row] = f.id;
    if (a.probs) a.probs[row] = (float)((double)f.w / (double)stays);
  }
}

void launch(const SampleArgs& a, hipStream_t s) { hipLaunchKernelGGL(k_sample_row, dim3(a.n_rows), dim3(ST), 0, s, a); }

}  // namespace

void launch_sample_decode(const float* logits, int32_t vocab, const float* d_uniform, const keep_sampling& how, int32_t* token,
                          float* prob, hipStream_t s) {
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
  launch(a, s);
}

}  // namespace keep

using namespace keep;

extern "C" uint64_t keep_sample_workspace_bytes(int32_t n_rows, int32_t vocab) {
  if (n_rows < 0 || n_rows > 65535 || vocab < 1 || vocab > KEEP_SAMPLE_MAX_VOCAB) return 0;
  return 256;
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
  const SampleArgs a{logits, d->row_stride, d->dtype, d->n_rows, d->vocab, uniform, temperature, top_k, top_p, min_p, 1.f, 1.f,
                     0.f, 0, -1, tokens, probs};
  launch(a, static_cast<hipStream_t>(stream));
  return launched(me);
}
