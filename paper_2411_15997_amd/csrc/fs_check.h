// Synchronous argument checks of the engine-step and cache operators' entry points (internal).
#pragma once
#include "fs_engine.h"

namespace fs {
namespace {

bool aligned_to(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) % n) == 0; }
bool mult8(int64_t x) { return (x & 7) == 0; }

fs_status status_of(hipError_t e) { return e == hipSuccess ? FS_OK : FS_E_HIP; }

int32_t rows_of(const fs_step *s) { return s->q_off_h[s->n_seqs]; }

fs_status check_step(const fs_step *s, bool lengths) {
  if (!s || s->n_seqs < 0 || s->n_seqs > 65535 || !s->q_off_h || s->q_off_h[0] != 0)
    return FS_E_ARG;
  for (int32_t i = 0; i < s->n_seqs; ++i)
    if (s->q_off_h[i + 1] < s->q_off_h[i]) return FS_E_ARG;
  if (rows_of(s) > (1 << 24)) return FS_E_ARG;
  if (rows_of(s) > 0 && !s->q_off) return FS_E_ARG;
  if (lengths && (s->max_kv < 0 || s->max_kv > (1 << 30) || (rows_of(s) > 0 && !s->kv_len)))
    return FS_E_ARG;
  return FS_OK;
}

fs_status check_cache(const fs_step *s, const fs_kv_cache *c, int32_t most_dim) {
  if (!c || (c->dtype != FS_BF16 && c->dtype != FS_F16)) return FS_E_ARG;
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024 || c->head_dim < 8 || c->head_dim > most_dim ||
      !mult8(c->head_dim))
    return FS_E_ARG;
  if (c->page_size < 1 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)))
    return FS_E_ARG;
  if (c->n_pages < 1 || c->n_pages > INT32_MAX) return FS_E_ARG;
  if (c->page_stride < 0 || c->head_stride < 0 || c->token_stride < 0 || !mult8(c->page_stride) ||
      !mult8(c->head_stride) || !mult8(c->token_stride) || c->page_stride > INT32_MAX ||
      c->head_stride > INT32_MAX || c->token_stride > INT32_MAX)
    return FS_E_ARG;
  // the offset inside a page, in elements, is computed in 32 bits
  if ((c->page_size - 1) * c->token_stride + (c->n_kv_heads - 1) * c->head_stride + c->head_dim >
      (int64_t(1) << 30))
    return FS_E_ARG;
  if (!aligned_to(c->k, 16) || !aligned_to(c->v, 16)) return FS_E_ARG;
  // the page table covers the longest length the step may hold
  if (c->table_stride < 0 ||
      (s->n_seqs > 0 && c->table_stride * c->page_size < int64_t(s->max_kv)))
    return FS_E_ARG;
  if (s->max_kv > 0 && rows_of(s) > 0 && (!c->k || !c->v || !c->table)) return FS_E_ARG;
  return FS_OK;
}

// What attention asks of a step, a cache of either kind (checked before) and its heads.
template <class Cache>
fs_status check_heads(const fs_step *s, const Cache *c, int32_t n_heads, int32_t window,
                      int32_t sinks) {
  if (c->head_dim != 64 && c->head_dim != 128) return FS_E_ARG;
  if (sinks < 0 || n_heads < 1 || n_heads % c->n_kv_heads || n_heads / c->n_kv_heads > 64 || window < 0)
    return FS_E_ARG;
  // keeps every count of work-items in 32 bits
  if (int64_t(rows_of(s)) * n_heads > (int64_t(1) << 30) ||
      int64_t(s->n_seqs) * c->n_kv_heads > (int64_t(1) << 20))
    return FS_E_ARG;
  return FS_OK;
}

fs_status check_attention(const fs_step *s, const fs_kv_cache *c, int32_t n_heads, int32_t window,
                          int32_t sinks) {
  fs_status st = check_step(s, true);
  if (st == FS_OK) st = check_cache(s, c, 128);
  if (st != FS_OK) return st;
  return check_heads(s, c, n_heads, window, sinks);
}

}  // namespace
}  // namespace fs
