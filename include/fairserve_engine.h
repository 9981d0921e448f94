/*
 * fairserve_engine.h -- the operators of one engine step (libfairserve.so, MI355X).
 *
 * The scheduler (fairserve.h) decides which calls an engine step prefills and decodes;
 * these entry points are what the step computes for them in a decoder layer and at its
 * end: a projection with every request's own low-rank adapter beside the shared weight,
 * rotary positions with the append to the paged KV cache, attention of the new tokens
 * over that cache, and the choice of the next token.
 *
 * Conventions are those of fairserve.h (device pointers unless the name ends in _h,
 * synchronous FS_E_ARG / FS_E_WORKSPACE, no allocation, no synchronisation, no pointer
 * kept, bit-deterministic results) with one difference: a step makes hundreds of these
 * calls, so they RAISE the device status word `err` and do not clear it.  One word
 * collects a whole step; the caller clears it with fs_clear_status before the step and
 * reads it with fs_sync_status after.  Every index read from device memory (page and
 * adapter ids, ranks, cached lengths) is checked before it is used as an address, so a wrong
 * one ends in FS_E_RANGE, not in a fault; outputs are unspecified after an error.  Not
 * checked is the device copy of fs_step's q_off, as little as that of fs_trace's rep_off: it
 * has to hold the host copy's values, from which grids and workspaces are sized.
 *
 * Every call may be captured into a HIP graph: what a replay may change is device data
 * (kv_len, the page table, adapter ids, sampling parameters); shapes, q_off and max_kv
 * are fixed by the capture.
 */
#ifndef FAIRSERVE_ENGINE_H
#define FAIRSERVE_ENGINE_H

#include "fairserve.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum fs_dtype { FS_BF16 = 0, FS_F16 = 1, FS_F32 = 2 } fs_dtype;

/* The requests of one engine step.  Request s brings the rows q_off[s] .. q_off[s+1]-1 of
 * the step's token matrices (a chunk of its prompt, one decoded token, or none).
 *   n_seqs   in [0, 65535]; at most 2^24 rows in all
 *   q_off_h  host   [n_seqs+1] int32, q_off_h[0] = 0, non-decreasing
 *   q_off    device [n_seqs+1] int32, same values (the caller's word: they are not compared)
 *   kv_len   device [n_seqs] int32: the request's tokens in the cache once this step's
 *            are appended; row i of its n rows has position kv_len - n + i.  A negative
 *            position marks a padding row: nothing is appended for it and its attention
 *            output is 0.  FS_E_RANGE unless 0 <= kv_len <= max_kv
 *   max_kv   host bound of every kv_len, at most 2^30 (sizes the work split, not the result) */
typedef struct fs_step {
  int32_t n_seqs;
  const int32_t *q_off_h;
  const int32_t *q_off;
  const int32_t *kv_len;
  int32_t max_kv;
} fs_step;

/* A paged KV cache of one layer.  Token p of request s lives in page
 * table[s * table_stride + p / page_size], slot p % page_size:
 *   k + page * page_stride + head * head_stride + slot * token_stride + d
 * and the same for v (strides in elements; d contiguous).  Pages may be shared between
 * requests (a common prompt prefix), in any order.  dtype FS_BF16 or FS_F16;
 * page_size a power of two in [1, 4096]; page ids in [0, n_pages), else FS_E_RANGE.
 * k, v and the strides must keep rows 16-byte aligned; strides below 2^31, a page's own rows
 * within 2^30 elements (a cache of any size).  Slots at and after kv_len are never used,
 * whatever they hold. */
typedef struct fs_kv_cache {
  int32_t dtype, n_kv_heads, head_dim, page_size;
  int64_t n_pages;
  void *k, *v;
  int64_t page_stride, head_stride, token_stride;
  const int32_t *table;
  int64_t table_stride;
} fs_kv_cache;

/* Clears a status word (a kernel on `stream`: may be captured). */
fs_status fs_clear_status(int32_t *err, hipStream_t stream);

/* y[t][n] = sum_k w[n][k] x[t][k] + scale[a] sum_{j < rank[a]} b[a][n][j] h[t][j],
 * h[t][j] = sum_k a[a][j][k] x[t][k], with a = adapter[s] of the request s that row t
 * belongs to (-1: the shared projection alone).
 *   x [T][K] (row stride x_stride), w [N][K], y [T][N] (row stride y_stride), all dtype
 *   (FS_BF16 or FS_F16); T = q_off_h[n_seqs]
 *   a [n_adapters][max_rank][K], b [n_adapters][N][max_rank]; entries at and after
 *   rank[a] are not used.  rank NULL: max_rank; scale NULL: 1
 * K, N, max_rank and the strides are multiples of 8, bases 16-byte aligned, max_rank <= 128,
 * K, N <= 2^20, x_stride <= 2^21,
 * n_adapters may be 0 (adapter is then not read).  Sums are held in fp32; scale * h enters the
 * second product as the sum of two dtype values (its rounding is below fp32's of the sum; in
 * FS_F16 in units of a power of two of the row's own, so that it may exceed the type's range).
 * What is not finite in one adapter reaches its own requests' rows alone.
 * ws: fs_adapter_workspace(s, ad) bytes, 256-byte aligned.  err: FS_E_RANGE for an
 * adapter outside [-1, n_adapters) or a rank outside [0, max_rank]. */
typedef struct fs_adapters {
  int32_t dtype, in_features, out_features, n_adapters, max_rank;
  const void *a, *b;
  const int32_t *rank;    /* device [n_adapters] or NULL */
  const float *scale;     /* device [n_adapters] or NULL */
  const int32_t *adapter; /* device [n_seqs] */
} fs_adapters;
size_t fs_adapter_workspace(const fs_step *s, const fs_adapters *ad);
fs_status fs_adapter_linear(const fs_step *s, const fs_adapters *ad, const void *x,
                            int64_t x_stride, const void *w, void *y, int64_t y_stride, void *ws,
                            size_t ws_bytes, int32_t *err, hipStream_t stream);

/* Rotary positions.  Pair i < rotary_dim/2 of a head turns by theta = p * inv_freq[i]
 * (the product and its reduction in fp64: exact enough at any position), cos and sin
 * multiplied by `factor`; elements from rotary_dim on are copied.
 *   interleaved 0: pair i is (x[i], x[i + rotary_dim/2]); 1: (x[2i], x[2i+1])
 *   pos  device [T] int32, or NULL: the row's cache position (padding rows: 0) */
typedef struct fs_rope {
  int32_t rotary_dim, interleaved;
  const float *inv_freq;
  float factor;
  const int32_t *pos;
} fs_rope;

/* Host helper: inv_freq_h[i] for i < rotary_dim/2, base theta0, and long-context scaling
 *   FS_ROPE_PLAIN   theta0^(-2i/rotary_dim)
 *   FS_ROPE_LINEAR  the plain one divided by `scale` (positions compressed)
 *   FS_ROPE_BASE    the plain one for the base theta0 * scale^(rotary_dim/(rotary_dim-2)):
 *                   the lowest frequency is divided by `scale`, the highest is kept
 *   FS_ROPE_PARTS   pair by pair: with t = original_len * f / 2 pi turns over the original
 *                   context, f is kept where t >= beta_fast, divided by `scale` where
 *                   t <= beta_slow, and a blend linear in t between; *factor_h =
 *                   0.1 ln(scale) + 1 (otherwise 1)
 * Computed in fp64, rounded once.  Synchronous. */
#define FS_ROPE_PLAIN 0
#define FS_ROPE_LINEAR 1
#define FS_ROPE_BASE 2
#define FS_ROPE_PARTS 3
fs_status fs_rope_frequencies(int32_t rotary_dim, double theta0, int32_t scaling, double scale,
                              int32_t original_len, double beta_fast, double beta_slow,
                              float *inv_freq_h, float *factor_h);

/* Turns the step's queries and keys and appends its keys and values to the cache.
 *   q [T][n_heads][head_dim] (token stride q_stride; heads contiguous) -> q_out (stride
 *   q_out_stride; may be q itself); k, v [T][n_kv_heads][head_dim] (strides k_stride,
 *   v_stride) -> the cache slots of the rows' positions.  All of the cache's dtype,
 *   head_dim a multiple of 8, at most 256; strides multiples of 8, bases 16-byte
 *   aligned.  rotary_dim even, in [0, head_dim].  n_heads may be 0 (q, q_out NULL).
 *   Rows are rounded once. */
fs_status fs_rope_append(const fs_step *s, const fs_kv_cache *c, const fs_rope *r,
                         int32_t n_heads, const void *q, int64_t q_stride, const void *k,
                         int64_t k_stride, const void *v, int64_t v_stride, void *q_out,
                         int64_t q_out_stride, int32_t *err, hipStream_t stream);

/* Attention of the step's rows over the cache.  Row t of request s at position p, head h
 * (key/value head h / (n_heads / n_kv_heads)):
 *   out[t][h] = sum_j softmax_j(scale * q[t][h] . k_j) v_j
 * over the cached tokens j <= p, j < kv_len and, with window > 0, j > p - window.  A row with no
 * such token gets 0 (lse -inf).  lse [T][n_heads] fp32 (NULL: not wanted) is
 * ln sum_j exp(scale q . k_j), which joins results over parts of a context: NaN where a score
 * is NaN, inf where one is inf and none is NaN (out is NaN in both).
 *   q, out: [T][n_heads][head_dim] of the cache's dtype (token strides q_stride,
 *   out_stride); head_dim 64 or 128; n_heads a multiple of n_kv_heads, at most 64 times it;
 *   rows times n_heads at most 2^30, n_seqs times n_kv_heads at most 2^20.
 * Scores, softmax statistics and sums are fp32; the probabilities enter the second
 * product as the sum of two values of the cache's dtype (requests of up to 32 rows times
 * query heads of a key/value head, unless others of the call have up to 64) or as one.
 * Keys and values that a row does not see do not reach it, whatever they hold.
 * ws: fs_attention_workspace(...) bytes, 256-byte aligned (may be NULL when that is 0). */
size_t fs_attention_workspace(const fs_step *s, const fs_kv_cache *c, int32_t n_heads,
                              int32_t window);
fs_status fs_paged_attention(const fs_step *s, const fs_kv_cache *c, int32_t n_heads, float scale,
                             int32_t window, const void *q, int64_t q_stride, void *out,
                             int64_t out_stride, float *lse, void *ws, size_t ws_bytes,
                             int32_t *err, hipStream_t stream);

/* The next token of each row from its logits and one given random number.
 * Order of a row's tokens: larger logit first, equal logits by lower id (-0 equals 0; NaN
 * counts as -inf).  With m the largest logit and T the temperature, in fp64,
 *   w_i = floor(2^40 * 2^(-(m - x_i) * log2(e) / T))       (2^40 where x_i = m)
 * are integers, so every sum below is exact and no order of addition shows:
 *   top-k  the first k tokens of the order (k <= 0 or k >= vocab: all)
 *   top-p  of those, a token stays while the weights before it sum to less than
 *          max(1, ceil(top_p * W)), W the sum over the top-k tokens (top_p >= 1: all)
 *   min-p  of those, w_i >= ceil(min_p * 2^40) stays (the first token always does)
 * and w_i > 0 always.  With S the sum over what stayed, the token is the first id (in
 * order of ids) whose running sum of kept weights exceeds min(floor(u * S), S - 1).
 * Temperature 0: the first token of the order.  A row without a logit above -inf:
 * token -1, logprob -inf, kept 0.
 *   logits [rows][vocab] dtype (row stride `stride` elements), vocab in [1, 2^20],
 *   rows at most 2^21
 *   temperature, top_p, min_p float, top_k int32: device [rows], each may be NULL
 *   (1, 1, 0, all); temperature finite and >= 0, top_p and min_p in [0, 1], u in [0, 1):
 *   FS_E_RANGE otherwise (NaN included), and token -1
 *   token [rows] int32; logprob [rows] float = ln(w_token / S) and kept [rows] int32, the
 *   number of tokens that stayed (each may be NULL)
 * ws: fs_sample_workspace(...) bytes, 256-byte aligned (may be NULL when that is 0). */
typedef struct fs_sampling {
  const float *temperature;
  const int32_t *top_k;
  const float *top_p, *min_p;
} fs_sampling;
size_t fs_sample_workspace(int32_t dtype, int32_t rows, int32_t vocab);
fs_status fs_sample(int32_t dtype, int32_t rows, int32_t vocab, const void *logits, int64_t stride,
                    const fs_sampling *p, const float *u, int32_t *token, float *logprob,
                    int32_t *kept, void *ws, size_t ws_bytes, int32_t *err, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif
