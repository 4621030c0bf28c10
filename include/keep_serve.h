/*
 * keep_serve.h -- C ABI of the operators that serve answers from a joined cache: rotary positions of other layouts and
 * scalings, a cache kept in pages (as it is or in 8 bits), attention of new tokens over those pages, and sampling.
 *
 * What keep.h leaves after a prefill is a contiguous cache and a greedy choice.  The calls here continue from there:
 * keep_rope_rows turns a chunk's queries and keys to their positions, keep_cache_write stores keys and values in pages
 * (keep_cache_read gives them back, as group blocks of a keep_prompt for instance), keep_paged_attention lets one or many
 * new tokens of a ragged batch attend to them, keep_sample picks the next tokens, and keep_decode_sampled is keep_decode
 * with that choice.
 *
 * Conventions (beside those of keep.h)
 *   - The calls without a context keep nothing between calls: no allocation, no state, no work after the stream's.  They
 *     launch kernels on `stream` (hipStream_t or NULL; the current device must be the stream's and hold every buffer) and do not
 *     wait for them, so they may be captured into a graph.  What varies from step to step (positions, slots, lengths, page
 *     tables, sampling parameters) is DEVICE memory and is read when the kernels run; what shapes a launch is in the
 *     descriptions, which are HOST memory and are read before the call returns.
 *   - A workspace is used from a call's first kernel to its last and holds nothing that a later call reads.  Calls that may
 *     overlap (two streams, two graphs) need a workspace each.
 *   - Contents of DEVICE arrays are not checked on the host.  Each call says what a value outside its range does; no value
 *     makes a kernel read or write outside the buffers described.
 *   - Buffers of 16-byte aligned addresses and strides are read in 16-byte pieces; others are taken where a call says so.
 *   - The text of a failure is at keep_last_error(NULL), for keep_decode_sampled at keep_last_error(ctx).
 */
#ifndef KEEP_SERVE_H
#define KEEP_SERVE_H

#include "keep.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- rotary positions -------------------------------------------------------------------------------------------
 * A head's first rot_dim values are rot_dim / 2 pairs; pair j of a row at position p is turned by the angle p * f_j:
 *   (x1, x2) -> (m (x1 cos - x2 sin), m (x2 cos + x1 sin)),   m: a factor on the rotated values, usually 1.
 * HALF pairs value j with value j + rot_dim / 2 (keep_prefill's pairing), INTERLEAVED value 2 j with value 2 j + 1.
 * Values from rot_dim on are left as they are. */
typedef enum { KEEP_ROPE_HALF = 0, KEEP_ROPE_INTERLEAVED = 1 } keep_rope_layout;

/* How the frequencies f_j = theta^(-2 j / rot_dim) change where a model reads past the length it was trained on.
 * LINEAR: f_j / factor.  BASE: theta is replaced by theta * factor^(rot_dim / (rot_dim - 2)), which leaves the fastest pair
 * and divides the slowest frequency by factor (a single pair is left).  PARTS: a pair that turns at least `fast` times over trained_len
 * positions is left, one that turns at most `slow` times is divided by factor, those between are mixed linearly in their
 * number of turns; the factor on rotated values becomes 0.1 ln(factor) + 1. */
typedef enum { KEEP_ROPE_PLAIN = 0, KEEP_ROPE_LINEAR = 1, KEEP_ROPE_BASE = 2, KEEP_ROPE_PARTS = 3 } keep_rope_scaling;

typedef struct {
  int32_t rot_dim;     /* even, >= 2 */
  int32_t scaling;     /* keep_rope_scaling */
  double theta;        /* > 0 */
  double factor;       /* >= 1; read by every scaling but PLAIN */
  int32_t trained_len; /* >= 1; read by PARTS */
  double fast, slow;   /* fast > slow >= 0; read by PARTS */
} keep_rope_desc;

/* freq: HOST [rot_dim / 2], radians per position, in the order of the pairs; magnitude: HOST scalar, m above.  Host
 * arithmetic in double.  Errors: INVALID_ARG. */
keep_status keep_rope_frequencies(const keep_rope_desc* desc, double* freq, float* magnitude);

typedef struct {
  int32_t dtype;                 /* keep_dtype of queries and keys */
  int32_t n_rows;                /* >= 0 */
  int32_t n_q_heads, n_kv_heads; /* heads of q and of k, each >= 0; not both 0 */
  int32_t head_dim;              /* 1 .. 1024 */
  int32_t rot_dim;               /* even, 2 .. head_dim */
  int32_t layout;                /* keep_rope_layout */
  float magnitude;
  /* elements from one row to the next; a row's heads are head_dim apart.  At least n_heads * head_dim. */
  int64_t q_in_stride, q_out_stride, k_in_stride, k_out_stride;
} keep_rope_rows_desc;

/* Turns the queries and keys of n_rows tokens.
 *   q_in, k_in -> q_out, k_out: DEVICE, any element-aligned address; out may be the in pointer itself (with the same stride),
 *     otherwise the two must not share an element (other columns of the same rows, with the same stride, are separate).  q_out
 *     must share none with k_in or k_out, nor q_in with k_out.  The pointers of q (of k) are not read when n_q_heads
 *     (n_kv_heads) is 0.
 *   positions: DEVICE int32 [n_rows], any value; a negative one turns back.
 *   freq: DEVICE double [rot_dim / 2].
 * Angles are formed and reduced in double, products in binary32, results rounded once.
 * Errors: INVALID_ARG (NULL, sizes, strides, overlap), SHAPE (head_dim), HIP. */
keep_status keep_rope_rows(const keep_rope_rows_desc* desc, const void* q_in, void* q_out, const void* k_in, void* k_out,
                           const int32_t* positions, const double* freq, void* stream);

/* ---- a cache in pages ------------------------------------------------------------------------------------------
 * Keys and values of page_size tokens make a page; which pages hold a sequence, and in which order, is the caller's
 * (a page table).  Slot s is token s % page_size of page s / page_size.
 * The 8-bit formats keep one binary32 scale per token and head, of keys and of values:
 *   scale = max(largest magnitude of the head_dim values * (1 / Q), 2^-126),   code = value / scale, at most Q in magnitude,
 * rounded to the nearest even code (INT8: whole numbers, Q = 127; FP8: the 8-bit floats of 4 exponent and 3 mantissa bits,
 * Q = 448), each operation rounded to binary32; a code stands for code * scale.  A head with a value that is not finite is
 * stored with the scale NaN and reads back as NaN throughout. */
typedef enum { KEEP_CACHE_F32 = 0, KEEP_CACHE_BF16 = 1, KEEP_CACHE_FP8 = 2, KEEP_CACHE_INT8 = 3 } keep_cache_format;

typedef struct {
  int32_t format; /* keep_cache_format */
  int32_t n_pages, page_size, n_kv_heads;
  int32_t head_dim; /* a multiple of 16, up to 256 */
  /* elements between pages, heads and tokens of k and of v (both laid out alike; a head's values are adjacent).  Each a
   * multiple of 16 bytes.  A page's values lie within its page_stride, its tokens and heads in either order.  Dense pages
   * [n_kv_heads][page_size][head_dim] keep a head's tokens together, which reads fastest; the joined cache of a prefill,
   * [tokens][n_kv_heads][head_dim], is the pages of token_stride = n_kv_heads * head_dim, head_stride = head_dim and
   * page_stride = page_size * token_stride. */
  int64_t page_stride, head_stride, token_stride;
  void *k, *v;             /* DEVICE, 16-byte aligned */
  float *k_scale, *v_scale; /* DEVICE [n_pages][n_kv_heads][page_size]; 8-bit formats only, else NULL */
} keep_paged_cache;

/* Stores the keys and values of n_rows tokens.
 *   k, v: DEVICE, dtype, row r at r * row_stride elements ([n_kv_heads][head_dim] each); 16-byte aligned, strides too.
 *   slots: DEVICE int32 [n_rows]; a slot outside [0, n_pages * page_size) drops its row (padding).  Rows of one call must
 *     have different slots: which of two rows with one slot stays, and whether codes and scale are of the same row, is not
 *     defined.
 * Errors: INVALID_ARG, SHAPE (head_dim, more than 2^31 - 1 slots), HIP. */
keep_status keep_cache_write(const keep_paged_cache* cache, int32_t dtype, const void* k, const void* v, int32_t n_rows,
                             int64_t row_stride, const int32_t* slots, void* stream);

/* Reads the keys and values of n_rows slots back as dtype (rounded to nearest even), row r to r * row_stride elements.
 * Rows whose slot is outside the cache are left as they were.  Otherwise as keep_cache_write. */
keep_status keep_cache_read(const keep_paged_cache* cache, int32_t dtype, void* k, void* v, int32_t n_rows,
                            int64_t row_stride, const int32_t* slots, void* stream);

/* ---- attention of new tokens over the pages -----------------------------------------------------------------------
 * Sequence s owns query rows q_start[s] .. q_start[s+1] - 1, its newest tokens, whose keys and values are in the cache
 * already: of kv_len[s] tokens in all they are the last, so the first of them sits at position kv_len[s] - (number of
 * rows).  A row sees the keys at positions up to its own, with a window w only the last w of those.  A row that sees
 * none (its position is negative) gets zeros and a log-sum-exp of -infinity. */
typedef struct {
  int32_t dtype;     /* keep_dtype of queries and output */
  int32_t n_seqs;    /* 0 .. KEEP_PAGED_MAX_SEQS */
  int32_t n_rows;    /* rows of q and out */
  int32_t n_q_heads; /* a multiple of the cache's n_kv_heads; query heads h * rep .. h * rep + rep - 1 read head h */
  int32_t max_pages; /* entries of a page table row, >= 1; max_pages * page_size <= 2^31 - 1024 */
  int32_t window;    /* 0: none */
  float scale;       /* factor on the scores; 0: 1 / sqrt(head_dim) */
  int64_t q_stride, out_stride; /* elements between rows, multiples of 16 bytes; heads are head_dim apart */
} keep_paged_attention_desc;
#define KEEP_PAGED_MAX_SEQS 4096

/* DEVICE bytes that keep_paged_attention needs for any lengths of such a cache with n_q_heads query heads and up to
 * n_seqs sequences; 0 if a description is invalid. */
uint64_t keep_paged_attention_workspace_bytes(const keep_paged_cache* cache, int32_t n_q_heads, int32_t n_seqs);

/*   q, out: DEVICE, 16-byte aligned, [n_rows] rows of [n_q_heads][head_dim]; they must not share an element (other columns of
 *     the same rows, with the same stride, are separate).
 *   q_start: DEVICE int32 [n_seqs + 1], not decreasing, within [0, n_rows] (clamped to that).  A sequence whose end lies
 *     before its start has no rows; what rows hold that two sequences claim is not defined.
 *   kv_len: DEVICE int32 [n_seqs] (clamped to [0, max_pages * page_size]).
 *   page_table: DEVICE int32 [n_seqs, max_pages]; entries behind a sequence's last page are not read, others are
 *     clamped to [0, n_pages).
 *   lse: DEVICE float [n_rows, n_q_heads] or NULL: log-sum-exp of each row's scaled scores.
 *   workspace: DEVICE, 256-byte aligned, at least keep_paged_attention_workspace_bytes.
 * Rows of out and lse that no sequence owns are left as they were.  A key or value that is not finite reaches only the
 * rows that see it.  Sums and statistics are binary32.  Their order depends on the two descriptions, q_start and kv_len (those
 * of all sequences: a launch's work is divided among workgroups by them), and in tiles with values that are not finite on
 * these; it does not depend on page numbers, contents of the workspace or timing.  So equal calls give equal bits, while other
 * neighbours in the batch, rows for padding or a wider page table can change a row's last bits.
 * bf16 queries with heads of 64, 128 or 256 over a bf16 or 8-bit cache (of less than 64 GB of keys) run on the bf16 matrix
 * instruction, with the probabilities rounded to bf16; everything else on the fp32 one.
 * Errors: INVALID_ARG, SHAPE, WORKSPACE (workspace_bytes too small), HIP. */
keep_status keep_paged_attention(const keep_paged_attention_desc* desc, const keep_paged_cache* cache, const void* q,
                                 const int32_t* q_start, const int32_t* kv_len, const int32_t* page_table, void* out,
                                 float* lse, void* workspace, uint64_t workspace_bytes, void* stream);

/* ---- sampling ------------------------------------------------------------------------------------------------------
 * One token per row of logits x, from a given uniform number u in [0, 1).  With the largest logit X, token i weighs
 *   w_i = rint(2^40 exp(-(X - x_i) / temperature))          (double arithmetic, a whole number)
 * so that every sum below is exact, whatever its order.  Tokens are ranked by logit, equal logits by the lower id first.
 *   min_p: a token stays if w_i >= ceil(min_p 2^40);   top_k: and if it ranks among the first top_k of those;
 *   top_p: and if the weights ranked before it sum to less than ceil(top_p * (sum of what stays so far)).
 * The token is the first in rank whose weights up to and with its own exceed floor(u * (sum of what stays)).  Both products
 * with a sum are double arithmetic, from the sum rounded to double (sums beyond 2^53 lose their last bits there).
 * Logits of NaN, and of -infinity beside larger ones, weigh nothing; +infinity outweighs everything finite.  Temperatures of 0
 * and below (and NaN) choose the largest logit, the lowest id among equals.  A row without a number above -infinity gets token -1
 * and probability 0. */
typedef struct {
  int32_t dtype;      /* keep_dtype of the logits */
  int32_t n_rows;     /* 0 .. 65535 */
  int32_t vocab;      /* 1 .. KEEP_SAMPLE_MAX_VOCAB */
  int64_t row_stride; /* elements between rows, >= vocab */
} keep_sample_desc;
#define KEEP_SAMPLE_MAX_VOCAB (1 << 20)

/* DEVICE bytes that keep_sample needs; 0 if n_rows or vocab is out of range. */
uint64_t keep_sample_workspace_bytes(int32_t n_rows, int32_t vocab);

/*   logits: DEVICE, element-aligned.  uniform: DEVICE float [n_rows], clamped to [0, 1).
 *   temperature, top_k, top_p, min_p: DEVICE [n_rows] each (float, int32, float, float), or NULL: 1, no limits.  top_k < 1,
 *     top_p >= 1 or NaN and min_p <= 0 or NaN are no limits; top_p <= 0 keeps the likeliest token, min_p > 1 counts as 1.
 *   tokens: DEVICE int32 [n_rows].  probs: DEVICE float [n_rows] or NULL: the token's share of what stayed.
 *   workspace: DEVICE, 256-byte aligned, at least keep_sample_workspace_bytes.
 * Errors: INVALID_ARG, SHAPE (vocab), WORKSPACE, HIP. */
keep_status keep_sample(const keep_sample_desc* desc, const void* logits, const float* uniform, const float* temperature,
                        const int32_t* top_k, const float* top_p, const float* min_p, int32_t* tokens, float* probs,
                        void* workspace, uint64_t workspace_bytes, void* stream);

typedef struct {
  float temperature;    /* 0 and below: greedy */
  int32_t top_k;        /* < 1: no limit */
  float top_p, min_p;   /* 1 and 0: no limits */
  const float* uniform; /* HOST [n_new], one number in [0, 1) per token */
} keep_sampling;

/* keep_decode with token t drawn as by keep_sample instead of the greedy choice (a row without a number above -infinity
 * gives token 0).  probs_out: HOST [n_new] or NULL.  Otherwise as keep_decode.
 * Errors: as keep_decode; INVALID_ARG for a NULL sampling or uniform, a uniform outside [0, 1), a temperature, top_p or
 * min_p that is not finite, SHAPE for a vocabulary above KEEP_SAMPLE_MAX_VOCAB. */
keep_status keep_decode_sampled(keep_ctx* ctx, const void* final_norm, const void* lm_head, const void* x_last,
                                void* k_cache, void* v_cache, int32_t cache_rows, int32_t n_ctx, int32_t n_new,
                                const keep_sampling* sampling, int32_t* tokens_out, float* probs_out, float* logits_out,
                                const int32_t* forced_tokens);

#ifdef __cplusplus
}
#endif
#endif /* KEEP_SERVE_H */
