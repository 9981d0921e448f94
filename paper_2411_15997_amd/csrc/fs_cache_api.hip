// extern "C" entry points of the cache's operators (declared in include/fairserve_cache.h):
// synchronous argument checks, then the launchers.
#include <cmath>

#include "fs_cache.h"
#include "fs_check.h"

namespace fs {
namespace {

bool in_31(int64_t x) { return x >= 0 && x <= INT32_MAX; }
bool is_row_type(int32_t dtype) { return dtype == FS_BF16 || dtype == FS_F16; }

// A 4-bit cache but for its table.
fs_status check_codes(const fs_kv_cache4 *c) {
  if (!c || c->n_kv_heads < 1 || c->n_kv_heads > 1024 || c->head_dim < 32 || c->head_dim > 256 ||
      c->head_dim % 32)
    return FS_E_ARG;
  if (c->page_size < 1 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)))
    return FS_E_ARG;
  if (c->n_pages < 1 || c->n_pages > INT32_MAX) return FS_E_ARG;
  if (!in_31(c->page_stride) || !in_31(c->head_stride) || !in_31(c->token_stride) ||
      (c->page_stride | c->head_stride | c->token_stride) & 15)
    return FS_E_ARG;
  if (!in_31(c->scale_page_stride) || !in_31(c->scale_head_stride) ||
      !in_31(c->scale_token_stride))
    return FS_E_ARG;
  // the offset inside a page is computed in 32 bits
  auto inside = [&](int64_t token, int64_t head, int64_t row) {
    return (c->page_size - 1) * token + (c->n_kv_heads - 1) * head + row;
  };
  if (inside(c->token_stride, c->head_stride, c->head_dim / 2) > (int64_t(1) << 30) ||
      inside(c->scale_token_stride, c->scale_head_stride, c->head_dim / 32) > (int64_t(1) << 30))
    return FS_E_ARG;
  if (!aligned_to(c->k, 16) || !aligned_to(c->v, 16)) return FS_E_ARG;
  return FS_OK;
}

fs_status check_cache4(const fs_step *s, const fs_kv_cache4 *c) {
  const fs_status st = check_codes(c);
  if (st != FS_OK) return st;
  // the page table covers the longest length the step may hold
  if (c->table_stride < 0 ||
      (s->n_seqs > 0 && c->table_stride * c->page_size < int64_t(s->max_kv)))
    return FS_E_ARG;
  if (s->max_kv > 0 && rows_of(s) > 0 &&
      (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->table))
    return FS_E_ARG;
  return FS_OK;
}

fs_status check_attention4(const fs_step *s, const fs_kv_cache4 *c, int32_t n_heads,
                           int32_t window, int32_t sinks) {
  fs_status st = check_step(s, true);
  if (st == FS_OK) st = check_cache4(s, c);
  if (st != FS_OK) return st;
  return check_heads(s, c, n_heads, window, sinks);
}

bool rows_ok(const void *p, int64_t stride, int64_t row) {
  return p && aligned_to(p, 16) && mult8(stride) && stride >= row;
}

fs_status check_pool(const fs_pages *p) {
  if (!p || p->n_pages < 1 || p->n_pages > (1 << 24) || p->page_size < 1 ||
      p->page_size > 4096 || (p->page_size & (p->page_size - 1)) || p->n_rows < 0 ||
      p->n_rows > 65535 || p->width < 0 || p->width > (1 << 30))
    return FS_E_ARG;
  if (!p->refs) return FS_E_ARG;
  if (p->n_rows > 0 && (!p->held || (p->width > 0 && !p->table) || p->table_stride < p->width))
    return FS_E_ARG;
  return FS_OK;
}

// Next to each other, tokens, then heads, become one piece.
void join(PageShape &s) {
  if (s.tokens == 1 || s.token_stride == s.bytes) {
    s.bytes *= s.tokens;
    s.tokens = 1;
    s.token_stride = s.bytes;
    if (s.heads == 1 || s.head_stride == s.bytes) {
      s.bytes *= s.heads;
      s.heads = 1;
    }
  }
}

}  // namespace
}  // namespace fs

using namespace fs;

extern "C" {

size_t fs_attention_sinks_workspace(const fs_step *s, const fs_kv_cache *c, int32_t n_heads,
                                    int32_t window, int32_t sinks) {
  if (check_attention(s, c, n_heads, window, sinks) != FS_OK) return 0;
  return attention_workspace_bytes(s, c, n_heads, window, sinks);
}

fs_status fs_paged_attention_sinks(const fs_step *s, const fs_kv_cache *c, int32_t n_heads,
                                   float scale, int32_t window, int32_t sinks, const void *q,
                                   int64_t q_stride, void *out, int64_t out_stride, float *lse,
                                   void *ws, size_t ws_bytes, int32_t *err, hipStream_t stream) {
  const fs_status st = check_attention(s, c, n_heads, window, sinks);
  if (st != FS_OK) return st;
  if (!err || !std::isfinite(scale)) return FS_E_ARG;
  if (rows_of(s) == 0) return FS_OK;
  const int64_t row = int64_t(n_heads) * c->head_dim;
  if (!rows_ok(q, q_stride, row) || !rows_ok(out, out_stride, row)) return FS_E_ARG;
  const size_t need = attention_workspace_bytes(s, c, n_heads, window, sinks);
  if (need > 0 && (!ws || !aligned_to(ws, 256) || ws_bytes < need)) return FS_E_WORKSPACE;
  return status_of(launch_attention(s, c, n_heads, scale, window, sinks, q, q_stride, out,
                                    out_stride, lse, ws, err, stream));
}

fs_status fs_rope_append4(const fs_step *s, const fs_kv_cache4 *c, const fs_rope *r, int32_t dtype,
                          int32_t n_heads, const void *q, int64_t q_stride, const void *k,
                          int64_t k_stride, const void *v, int64_t v_stride, void *q_out,
                          int64_t q_out_stride, int32_t *err, hipStream_t stream) {
  fs_status st = check_step(s, true);
  if (st == FS_OK) st = check_cache4(s, c);
  if (st != FS_OK) return st;
  if (!r || !err || !is_row_type(dtype) || r->rotary_dim < 0 || r->rotary_dim > c->head_dim ||
      (r->rotary_dim & 1) || r->interleaved < 0 || r->interleaved > 1 ||
      (r->rotary_dim > 0 && !r->inv_freq) || n_heads < 0 || n_heads > 65535)
    return FS_E_ARG;
  if (rows_of(s) == 0) return FS_OK;
  const int64_t row = int64_t(c->n_kv_heads) * c->head_dim, qrow = int64_t(n_heads) * c->head_dim;
  if (!rows_ok(k, k_stride, row) || !rows_ok(v, v_stride, row)) return FS_E_ARG;
  if (n_heads > 0 && (!rows_ok(q, q_stride, qrow) || !rows_ok(q_out, q_out_stride, qrow)))
    return FS_E_ARG;
  return status_of(launch_rope_append4(s, c, r, dtype, n_heads, q, q_stride, k, k_stride, v,
                                       v_stride, q_out, q_out_stride, err, stream));
}

fs_status fs_cache4_rows(const fs_step *s, const fs_kv_cache4 *c, int32_t dtype, void *k_out,
                         int64_t k_stride, void *v_out, int64_t v_stride, int32_t *err,
                         hipStream_t stream) {
  fs_status st = check_step(s, true);
  if (st == FS_OK) st = check_cache4(s, c);
  if (st != FS_OK) return st;
  if (!err || !is_row_type(dtype)) return FS_E_ARG;
  const int64_t row = int64_t(c->n_kv_heads) * c->head_dim;
  if ((k_out && !rows_ok(k_out, k_stride, row)) || (v_out && !rows_ok(v_out, v_stride, row)))
    return FS_E_ARG;
  if (rows_of(s) == 0 || (!k_out && !v_out)) return FS_OK;
  return status_of(
      launch_cache4_rows(s, c, dtype, k_out, k_stride, v_out, v_stride, err, stream));
}

size_t fs_attention4_workspace(const fs_step *s, const fs_kv_cache4 *c, int32_t n_heads,
                               int32_t window, int32_t sinks) {
  if (check_attention4(s, c, n_heads, window, sinks) != FS_OK) return 0;
  return attention4_workspace_bytes(s, c, n_heads, window, sinks);
}

fs_status fs_paged_attention4(const fs_step *s, const fs_kv_cache4 *c, int32_t dtype,
                              int32_t n_heads, float scale, int32_t window, int32_t sinks,
                              const void *q, int64_t q_stride, void *out, int64_t out_stride,
                              float *lse, void *ws, size_t ws_bytes, int32_t *err,
                              hipStream_t stream) {
  const fs_status st = check_attention4(s, c, n_heads, window, sinks);
  if (st != FS_OK) return st;
  if (!err || !is_row_type(dtype) || !std::isfinite(scale)) return FS_E_ARG;
  if (rows_of(s) == 0) return FS_OK;
  const int64_t row = int64_t(n_heads) * c->head_dim;
  if (!rows_ok(q, q_stride, row) || !rows_ok(out, out_stride, row)) return FS_E_ARG;
  const size_t need = attention4_workspace_bytes(s, c, n_heads, window, sinks);
  if (need > 0 && (!ws || !aligned_to(ws, 256) || ws_bytes < need)) return FS_E_WORKSPACE;
  return status_of(launch_attention4(s, c, dtype, n_heads, scale, window, sinks, q, q_stride, out,
                                     out_stride, lse, ws, err, stream));
}

fs_status fs_pages_free(const fs_pages *p, int32_t n, const int32_t *rows, int32_t *err,
                        hipStream_t stream) {
  const fs_status st = check_pool(p);
  if (st != FS_OK) return st;
  if (n < 0 || !err || (n > 0 && !rows)) return FS_E_ARG;
  if (n == 0) return FS_OK;
  return status_of(launch_pages_free(p, n, rows, err, stream));
}

size_t fs_pages_workspace(const fs_pages *p, int32_t n) {
  if (check_pool(p) != FS_OK || n < 0 || n > 65535) return 0;
  return pages_workspace_bytes(p, n);
}

fs_status fs_pages_fork(const fs_pages *p, int32_t n, const int32_t *parent, const int32_t *child,
                        const int32_t *shared, const int32_t *room, int32_t *src, int32_t *dst,
                        void *ws, size_t ws_bytes, int32_t *err, hipStream_t stream) {
  const fs_status st = check_pool(p);
  if (st != FS_OK) return st;
  if (n < 0 || n > 65535 || !err) return FS_E_ARG;
  if (n == 0) return FS_OK;
  if (!parent || !child || !shared || !room || !src || !dst) return FS_E_ARG;
  if (!ws || !aligned_to(ws, 256) || ws_bytes < pages_workspace_bytes(p, n)) return FS_E_WORKSPACE;
  return status_of(
      launch_pages_fork(p, n, parent, child, shared, room, src, dst, ws, err, stream));
}

fs_status fs_pages_compact(const fs_pages *p, int32_t *refs_out, int32_t *table_out,
                           int64_t table_out_stride, int32_t *src, int32_t *dst, int32_t *count,
                           void *ws, size_t ws_bytes, int32_t *err, hipStream_t stream) {
  const fs_status st = check_pool(p);
  if (st != FS_OK) return st;
  if (!err || !refs_out || !count || (p->n_pages > 1 && (!src || !dst))) return FS_E_ARG;
  if (p->n_rows > 0 && ((p->width > 0 && !table_out) || table_out_stride < p->width))
    return FS_E_ARG;
  if (table_out == p->table && p->n_rows > 1 && table_out_stride != p->table_stride)
    return FS_E_ARG;
  if (!ws || !aligned_to(ws, 256) || ws_bytes < pages_workspace_bytes(p, 0)) return FS_E_WORKSPACE;
  return status_of(launch_pages_compact(p, refs_out, table_out, table_out_stride, src, dst, count,
                                        ws, err, stream));
}

fs_status fs_pages_copy(const fs_kv_cache *layers, int32_t n_layers, int32_t n, const int32_t *src,
                        const int32_t *dst, const int32_t *count, int32_t *err,
                        hipStream_t stream) {
  if (n_layers < 0 || n_layers > 65536 || n < 0 || n > (1 << 24) || !err) return FS_E_ARG;
  if (n_layers == 0 || n == 0) return FS_OK;
  if (!layers || !src || !dst) return FS_E_ARG;
  const fs_kv_cache &c = layers[0];
  const fs_step none = {};  // (its checks of a cache without a step's)
  for (int32_t i = 0; i < n_layers; ++i) {
    const fs_kv_cache &x = layers[i];
    const int32_t zero = 0;
    fs_step s = none;
    s.q_off_h = &zero;
    if (check_cache(&s, &x, 256) != FS_OK || !x.k || !x.v) return FS_E_ARG;
    if (x.dtype != c.dtype || x.n_kv_heads != c.n_kv_heads || x.head_dim != c.head_dim ||
        x.page_size != c.page_size || x.n_pages != c.n_pages || x.page_stride != c.page_stride ||
        x.head_stride != c.head_stride || x.token_stride != c.token_stride)
      return FS_E_ARG;
  }
  PageShape shape = {2 * c.page_stride,     uint32_t(c.n_kv_heads), uint32_t(c.page_size),
                     uint32_t(2 * c.head_dim), 2 * c.head_stride,   2 * c.token_stride};
  join(shape);
  for (int32_t l = 0; l < n_layers; l += kLayers) {
    const int32_t m = n_layers - l < kLayers ? n_layers - l : kLayers;
    PageArrays a = {};
    for (int32_t i = 0; i < m; ++i) {
      a.at[i][0] = static_cast<char *>(layers[l + i].k);
      a.at[i][1] = static_cast<char *>(layers[l + i].v);
    }
    const hipError_t e = launch_pages_copy(a, m, 2, shape, shape, int32_t(c.n_pages), n, src, dst,
                                           count, err, stream);
    if (e != hipSuccess) return FS_E_HIP;
  }
  return FS_OK;
}

fs_status fs_pages_copy4(const fs_kv_cache4 *layers, int32_t n_layers, int32_t n,
                         const int32_t *src, const int32_t *dst, const int32_t *count,
                         int32_t *err, hipStream_t stream) {
  if (n_layers < 0 || n_layers > 65536 || n < 0 || n > (1 << 24) || !err) return FS_E_ARG;
  if (n_layers == 0 || n == 0) return FS_OK;
  if (!layers || !src || !dst) return FS_E_ARG;
  const fs_kv_cache4 &c = layers[0];
  for (int32_t i = 0; i < n_layers; ++i) {
    const fs_kv_cache4 &x = layers[i];
    if (check_codes(&x) != FS_OK || !x.k || !x.v || !x.k_scale || !x.v_scale) return FS_E_ARG;
    if (x.n_kv_heads != c.n_kv_heads || x.head_dim != c.head_dim || x.page_size != c.page_size ||
        x.n_pages != c.n_pages || x.page_stride != c.page_stride ||
        x.head_stride != c.head_stride || x.token_stride != c.token_stride ||
        x.scale_page_stride != c.scale_page_stride ||
        x.scale_head_stride != c.scale_head_stride ||
        x.scale_token_stride != c.scale_token_stride)
      return FS_E_ARG;
  }
  PageShape codes = {c.page_stride,        uint32_t(c.n_kv_heads), uint32_t(c.page_size),
                     uint32_t(c.head_dim / 2), c.head_stride,      c.token_stride};
  PageShape scales = {c.scale_page_stride,  uint32_t(c.n_kv_heads), uint32_t(c.page_size),
                      uint32_t(c.head_dim / 32), c.scale_head_stride, c.scale_token_stride};
  join(codes);
  join(scales);
  for (int32_t l = 0; l < n_layers; l += kLayers) {
    const int32_t m = n_layers - l < kLayers ? n_layers - l : kLayers;
    PageArrays a = {};
    for (int32_t i = 0; i < m; ++i) {
      a.at[i][0] = static_cast<char *>(layers[l + i].k);
      a.at[i][1] = static_cast<char *>(layers[l + i].v);
      a.at[i][2] = static_cast<char *>(layers[l + i].k_scale);
      a.at[i][3] = static_cast<char *>(layers[l + i].v_scale);
    }
    const hipError_t e = launch_pages_copy(a, m, 4, codes, scales, int32_t(c.n_pages), n, src, dst,
                                           count, err, stream);
    if (e != hipSuccess) return FS_E_HIP;
  }
  return FS_OK;
}

}  // extern "C"
