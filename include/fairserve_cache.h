/*
 * fairserve_cache.h -- operators of the KV cache beside those of fairserve_engine.h
 * (libfairserve.so, MI355X): a window whose first tokens stay visible, a cache held in 4
 * bits, and the pages that the requests of a cache share.
 *
 * Conventions are those of fairserve_engine.h: the calls RAISE the device status word and do
 * not clear it, check every index read from device memory before it becomes an address, may
 * be captured into a HIP graph, and leave rows and slots that they do not name as they were.
 */
#ifndef FAIRSERVE_CACHE_H
#define FAIRSERVE_CACHE_H

#include "fairserve_engine.h"

#ifdef __cplusplus
extern "C" {
#endif

/* fs_paged_attention with a window that leaves the first `sinks` tokens of a request visible:
 * the sum is over the cached tokens j <= p, j < kv_len with j > p - window or j < sinks.
 * sinks >= 0 (0, or window 0: fs_paged_attention itself).  Tokens keep the positions at which
 * they were appended. */
size_t fs_attention_sinks_workspace(const fs_step *s, const fs_kv_cache *c, int32_t n_heads,
                                    int32_t window, int32_t sinks);
fs_status fs_paged_attention_sinks(const fs_step *s, const fs_kv_cache *c, int32_t n_heads,
                                   float scale, int32_t window, int32_t sinks, const void *q,
                                   int64_t q_stride, void *out, int64_t out_stride, float *lse,
                                   void *ws, size_t ws_bytes, int32_t *err, hipStream_t stream);

/* A paged KV cache held in 4 bits: 4.25 bits a value.  A token's head is head_dim / 32 groups
 * of 32 neighbouring values.  A group has a scale byte b, which stands for 2^(b - 127), and
 * each value a code of 4 bits: bit 3 its sign, bits 0 to 2 one of 0, 0.5, 1, 1.5, 2, 3, 4, 6.
 * Value d of the group is in byte d / 2, low half first.  Token p of request s lives in page
 * table[s * table_stride + p / page_size], slot p % page_size:
 *   codes   k + page * page_stride + head * head_stride + slot * token_stride + d / 2
 *   scales  k_scale + page * scale_page_stride + head * scale_head_stride
 *                   + slot * scale_token_stride + d / 32
 * and the same for v and v_scale (strides in bytes; a head's codes and scales contiguous).
 * head_dim a multiple of 32, at most 256; k, v and their strides 16-byte aligned (scales need
 * no alignment); strides below 2^31, a page's own rows within 2^30 bytes; pages, page ids and
 * the table as in fs_kv_cache.
 * Rows of dtype FS_BF16 or FS_F16 go in and come out.  A scale byte of 0 counts as 1; one above
 * 252 (FS_BF16) or 140 (FS_F16), whose codes could leave that type's range, as NaN for all 32
 * values. */
typedef struct fs_kv_cache4 {
  int32_t n_kv_heads, head_dim, page_size;
  int64_t n_pages;
  void *k, *v;
  int64_t page_stride, head_stride, token_stride;
  void *k_scale, *v_scale;
  int64_t scale_page_stride, scale_head_stride, scale_token_stride;
  const int32_t *table;
  int64_t table_stride;
} fs_kv_cache4;

/* fs_rope_append into a cache of 4 bits: queries are turned into q_out, keys are turned and
 * keys and values appended.  q, k, v, q_out of `dtype`, laid out and aligned as there.
 * A group x of 32 values takes the scale 2^E with the least E for which max |x| <= 7 * 2^E (so
 * that no value is off by more than 2^E, half of the widest step), E + 127 held to 1 .. 252
 * (FS_F16: 1 .. 140), and each value the code nearest to x / 2^E (ties to the even code, at
 * most 6).  A group with a value that is not finite takes the scale byte 255.  Keys are turned
 * in fp64 and rounded to fp32 before: a code does not hang on the order of operations. */
fs_status fs_rope_append4(const fs_step *s, const fs_kv_cache4 *c, const fs_rope *r, int32_t dtype,
                          int32_t n_heads, const void *q, int64_t q_stride, const void *k,
                          int64_t k_stride, const void *v, int64_t v_stride, void *q_out,
                          int64_t q_out_stride, int32_t *err, hipStream_t stream);

/* What the cache holds at the positions of the step's rows, as values of `dtype`:
 * k_out, v_out [T][n_kv_heads][head_dim] (token strides in elements, multiples of 8; bases
 * 16-byte aligned; each may be NULL).  Padding rows (negative positions) and rows of a length
 * out of range are 0. */
fs_status fs_cache4_rows(const fs_step *s, const fs_kv_cache4 *c, int32_t dtype, void *k_out,
                         int64_t k_stride, void *v_out, int64_t v_stride, int32_t *err,
                         hipStream_t stream);

/* fs_paged_attention over a cache of 4 bits, with a window and sinks as above; q and out of
 * `dtype`.  head_dim 64 or 128 and the other limits as there.  The values that codes and
 * scales stand for are exact in `dtype` (FS_F16: in its range); the rest is as in
 * fs_paged_attention, the rounding of the probabilities included.  A group of the cache that
 * counts as NaN makes out and lse of the rows that see it NaN (k), or its 32 values of out (v);
 * a query with a value that is not finite reaches its own row alone.  Sums stay finite while
 * |v| < 2^100 (FS_BF16). */
size_t fs_attention4_workspace(const fs_step *s, const fs_kv_cache4 *c, int32_t n_heads,
                               int32_t window, int32_t sinks);
fs_status fs_paged_attention4(const fs_step *s, const fs_kv_cache4 *c, int32_t dtype,
                              int32_t n_heads, float scale, int32_t window, int32_t sinks,
                              const void *q, int64_t q_stride, void *out, int64_t out_stride,
                              float *lse, void *ws, size_t ws_bytes, int32_t *err,
                              hipStream_t stream);

/* The pages of a cache and the rows of its page table that hold them.  One pool serves all
 * layers' caches of that table.
 *   refs  device [n_pages]  how many rows hold the page (0: it is free); a caller that keeps
 *         a page of its own adds one
 *   table device [n_rows][width] page ids (row stride table_stride >= width; rows do not
 *         overlap); held device [n_rows]: row s holds the pages table[s][0 .. held[s] - 1].
 *         Entries from held[s] on are not used and left as they were.
 * page_size a power of two in [1, 4096], n_rows in [0, 65535], width in [0, 2^30],
 * n_pages in [1, 2^24], else FS_E_ARG.  FS_E_RANGE for a row outside [0, n_rows), a held
 * outside [0, width], a page id outside [0, n_pages) among the held. */
typedef struct fs_pages {
  int32_t n_pages, page_size, n_rows, width;
  int32_t *refs, *table, *held;
  int64_t table_stride;
} fs_pages;

/* Lets go of all pages of the rows rows[0 .. n-1] (device): each page's refs goes down by one
 * for each row that held it, held becomes 0.  A row named twice is let go once.  FS_E_RANGE,
 * and a refs that stays 0, for a held page that is free. */
fs_status fs_pages_free(const fs_pages *p, int32_t n, const int32_t *rows, int32_t *err,
                        hipStream_t stream);

/* Gives the rows child[0 .. n-1] (device; n at most 65,535), which hold nothing, their pages.
 * Row child[i] begins with the first shared[i] tokens of row parent[i] (-1: none, shared[i] 0)
 * and gets room for room[i] >= shared[i] tokens: the parent's floor(shared / page_size) whole
 * pages, whose refs go up by one, then free pages, the lowest ids first in order of i.  Where
 * shared is no multiple of page_size the first new page is a copy of the parent's next one,
 * to be made in each layer by fs_pages_copy: src[i] -> dst[i] (otherwise both -1).
 * So a page that is held twice is whole and is not written again.
 * Parents and free pages are those before the call.  FS_E_RANGE, and no pages, src = dst = -1
 * for the i in question, the others getting theirs as if it were not there: a parent, child or
 * length out of range, a child that holds pages or is named by a lower i, a parent that does
 * not hold the shared tokens, a page id out of range or a free page among the shared ones, a
 * room beyond width pages.  FS_E_OVERFLOW, and nothing at all is given, where the free pages do
 * not suffice.
 * ws: fs_pages_workspace(p, n) bytes, 256-byte aligned; so for fs_pages_compact (n = 0). */
size_t fs_pages_workspace(const fs_pages *p, int32_t n);
fs_status fs_pages_fork(const fs_pages *p, int32_t n, const int32_t *parent, const int32_t *child,
                        const int32_t *shared, const int32_t *room, int32_t *src, int32_t *dst,
                        void *ws, size_t ws_bytes, int32_t *err, hipStream_t stream);

/* Moves the L pages in use (refs > 0) into ids 0 .. L - 1: the i-th in-use page with an id
 * >= L moves to the i-th free id < L, src[i] -> dst[i], i < *count <= n_pages / 2; src and dst
 * [n_pages / 2] are -1 from *count on.  refs_out [n_pages] and table_out (row stride
 * table_out_stride >= width, entries from held on left as they were) get the new ids; each
 * may be the pool's own, and else does not overlap it.  FS_E_RANGE for a held page that is free,
 * whose entry keeps its id (other contents may move there).  The pages' contents are moved in
 * each layer by fs_pages_copy. */
fs_status fs_pages_compact(const fs_pages *p, int32_t *refs_out, int32_t *table_out,
                           int64_t table_out_stride, int32_t *src, int32_t *dst, int32_t *count,
                           void *ws, size_t ws_bytes, int32_t *err, hipStream_t stream);

/* Copies page src[i] to page dst[i] in k and v (scales included) of n_layers caches,
 * i < min(n, *count) (count device, NULL: n); pairs of -1 are passed over.  `layers` is a host
 * array of caches (head_dim at most 256) alike in all but their k, v (and scale) addresses
 * (their tables are not read), n_layers in [0, 2^16], n in [0, 2^24].
 * No dst may be another pair's src or dst, else those pages' contents are unspecified.
 * FS_E_RANGE for an id outside [-1, n_pages) or a pair with one -1. */
fs_status fs_pages_copy(const fs_kv_cache *layers, int32_t n_layers, int32_t n, const int32_t *src,
                        const int32_t *dst, const int32_t *count, int32_t *err,
                        hipStream_t stream);
fs_status fs_pages_copy4(const fs_kv_cache4 *layers, int32_t n_layers, int32_t n,
                         const int32_t *src, const int32_t *dst, const int32_t *count,
                         int32_t *err, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif
