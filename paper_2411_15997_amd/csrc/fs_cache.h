// Shared by the operators of the 4-bit cache and of its pages (internal): the 4-bit format as
// kernels read it, and the host-side launchers.
#pragma once
#include "../../include/fairserve_cache.h"
#include "fs_engine.h"

namespace fs {

// The scales of a 4-bit cache (strides in bytes); its codes are a DevCache in bytes.
struct DevScales {
  const uint8_t *k, *v;
  uint32_t page_stride, head_stride, token_stride;
};

inline DevCache dev_codes(const fs_kv_cache4 *c) {
  DevCache d;
  d.k = static_cast<const char *>(c->k);
  d.v = static_cast<const char *>(c->v);
  d.page_stride = uint32_t(c->page_stride);
  d.head_stride = uint32_t(c->head_stride);
  d.token_stride = uint32_t(c->token_stride);
  d.n_pages = uint32_t(c->n_pages);
  d.table = c->table;
  d.table_stride = c->table_stride;
  d.page_shift = __builtin_ctz(unsigned(c->page_size));
  d.n_kv_heads = c->n_kv_heads;
  d.head_dim = c->head_dim;
  return d;
}
inline DevScales dev_scales(const fs_kv_cache4 *c) {
  DevScales d;
  d.k = static_cast<const uint8_t *>(c->k_scale);
  d.v = static_cast<const uint8_t *>(c->v_scale);
  d.page_stride = uint32_t(c->scale_page_stride);
  d.head_stride = uint32_t(c->scale_head_stride);
  d.token_stride = uint32_t(c->scale_token_stride);
  return d;
}

// The largest scale byte whose codes (up to 6) stay in the type's range: 6 * 2^125 and 6 * 2^13.
template <bool BF>
constexpr uint32_t kTopScale = BF ? 252 : 140;

// The power of two of a scale byte; 1 where the group counts as NaN (its codes are then not
// used, but have to stay finite where a product meets them).
template <bool BF>
__device__ inline float scale_of(uint32_t byte) {
  const uint32_t b = byte > kTopScale<BF> ? 127 : byte;
  return __uint_as_float((b > 1 ? b : 1) << 23);
}

// The eight values of a word of codes, times the scale: exact in the 16-bit type.
template <bool BF>
__device__ inline s16x8 values8(uint32_t codes, float scale) {
  typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
  u32x4 w;
  if constexpr (BF) {
    w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  } else {
    w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 0));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 1));
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 2));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 3));
  }
  return __builtin_bit_cast(s16x8, w);
}

// ---- launchers
hipError_t launch_rope_append4(const fs_step *s, const fs_kv_cache4 *c, const fs_rope *r,
                               int32_t dtype, int32_t n_heads, const void *q, int64_t q_stride,
                               const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                               void *q_out, int64_t q_out_stride, int32_t *err,
                               hipStream_t stream);
hipError_t launch_cache4_rows(const fs_step *s, const fs_kv_cache4 *c, int32_t dtype, void *k_out,
                              int64_t k_stride, void *v_out, int64_t v_stride, int32_t *err,
                              hipStream_t stream);

size_t attention4_workspace_bytes(const fs_step *s, const fs_kv_cache4 *c, int32_t n_heads,
                                  int32_t window, int32_t sinks);
hipError_t launch_attention4(const fs_step *s, const fs_kv_cache4 *c, int32_t dtype,
                             int32_t n_heads, float scale, int32_t window, int32_t sinks,
                             const void *q, int64_t q_stride, void *out, int64_t out_stride,
                             float *lse, void *ws, int32_t *err, hipStream_t stream);

size_t pages_workspace_bytes(const fs_pages *p, int32_t n);
hipError_t launch_pages_free(const fs_pages *p, int32_t n, const int32_t *rows, int32_t *err,
                             hipStream_t stream);
hipError_t launch_pages_fork(const fs_pages *p, int32_t n, const int32_t *parent,
                             const int32_t *child, const int32_t *shared, const int32_t *room,
                             int32_t *src, int32_t *dst, void *ws, int32_t *err,
                             hipStream_t stream);
hipError_t launch_pages_compact(const fs_pages *p, int32_t *refs_out, int32_t *table_out,
                                int64_t table_out_stride, int32_t *src, int32_t *dst,
                                int32_t *count, void *ws, int32_t *err, hipStream_t stream);

// One of the arrays of a cache as pages are copied: `rows` x `tokens` pieces of `bytes`, their
// strides in bytes (pieces next to each other are joined before).
struct PageShape {
  int64_t page_stride;
  uint32_t heads, tokens, bytes;
  int64_t head_stride, token_stride;
};
constexpr int kLayers = 48;  // of one launch: their addresses are kernel arguments
struct PageArrays {
  char *at[kLayers][4];  // k, v, and the scales of a 4-bit cache
};
hipError_t launch_pages_copy(const PageArrays &arrays, int32_t n_layers, int32_t n_kinds,
                             const PageShape &codes, const PageShape &scales, int32_t n_pages,
                             int32_t n, const int32_t *src, const int32_t *dst,
                             const int32_t *count, int32_t *err, hipStream_t stream);

}  // namespace fs
