// Shared by the engine-step operators (internal): 16-bit types, the step's rows, and the
// host-side launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/fairserve_engine.h"
#include "fs_device.h"

namespace fs {

typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;

// The two 16-bit types: BF selects bfloat16, else IEEE half.  Stores round to nearest even.
template <bool BF>
struct T16;
template <>
struct T16<true> {
  typedef __bf16 E;
  typedef bf16x8 V8;
};
template <>
struct T16<false> {
  typedef _Float16 E;
  typedef f16x8 V8;
};
template <bool BF>
__device__ inline float to_f32(short x) {
  return float(__builtin_bit_cast(typename T16<BF>::E, x));
}
template <bool BF>
__device__ inline short to_16(float x) {
  return __builtin_bit_cast(short, typename T16<BF>::E(x));
}

// D = A B + C on the matrix cores (A: rows, B: columns, 8 consecutive k per lane).
template <bool BF>
__device__ inline f32x4 mfma_16x16x32(s16x8 a, s16x8 b, f32x4 c) {
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <bool BF>
__device__ inline f32x16 mfma_32x32x16(s16x8 a, s16x8 b, f32x16 c) {
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// 16 bytes for each lane from `base` (the same for the wave) plus its own offset in bytes
// straight into LDS, at address `at` (the same for the wave) plus 16 times the lane.
// Counted by vmcnt, in order; wait_loads() before use.  Written out because the compiler
// would wait for all such loads before any LDS read.  No register is loaded: nothing of
// the wave's own can be overwritten while it is under way.
// (m0 is reserved: the compiler keeps no value of its own there from one statement to the
// next, and wants it on no list of clobbered registers.)
__device__ inline void load_to_lds(const void *base, uint32_t offset, uint32_t at) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(at),
               "v"(offset), "s"(base)
               : "memory");
}
// The same from each lane's own 64-bit address.
__device__ inline void load_to_lds(const void *from, uint32_t at) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(at), "v"(from)
               : "memory");
}
__device__ inline uint32_t lds_address(const void *p) {
  return __builtin_amdgcn_readfirstlane(
      uint32_t(uintptr_t((__attribute__((address_space(3))) const void *)p)));
}
// Waits until at most LEFT of the wave's newest loads are under way and its LDS reads are
// done, then for the other waves: what they loaded is there, what they read may be replaced.
template <int LEFT>
__device__ inline void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// The same for a wave that reads only what it loaded itself: reads_done() before a buffer
// is loaded again, wait_own() before one is read.
__device__ inline void reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
template <int LEFT>
__device__ inline void wait_own() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
}

// The last of the requests 0 .. n - 1 whose first(s) is at most b, by the whole wave: 64
// probes a round instead of one.  first is non-decreasing and first(0) <= b.  All 64 lanes
// take part, with the same b: lanes that have left, or that look for another b, would make
// the count of hits wrong.
template <class F>
__device__ inline int32_t last_at_most(int32_t n, int32_t b, F first) {
  int32_t lo = 0, len = n;
  while (len > 1) {
    const int32_t step = (len + 63) >> 6, at = int32_t(__lane_id()) * step;
    const int32_t hits = __popcll(__ballot(at < len && first(lo + at) <= b));
    const int32_t from = lo + (hits - 1) * step;
    len = min(step, lo + len - from);
    lo = from;
  }
  return lo;
}
// The request whose rows contain row t (t < q_off[n]), by the whole wave (one t for all 64
// lanes).
__device__ inline int32_t seq_of_row(const int32_t *q_off, int32_t n, int32_t t) {
  return last_at_most(n, t, [&](int32_t s) { return __ldg(q_off + s); });
}
// The same by each lane for a t of its own, whatever the other lanes do.
__device__ inline int32_t seq_of_own_row(const int32_t *q_off, int32_t n, int32_t t) {
  int32_t lo = 0, hi = n - 1;
  while (lo < hi) {
    const int32_t mid = (lo + hi + 1) >> 1;
    if (__ldg(q_off + mid) <= t)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

// Row tiles that never span two requests.  Request s owns the tile numbers from
// (q_off[s] >> SHIFT) + s on: at least as many as its rows need, so the whole step fits
// (q_off[n] >> SHIFT) + n numbers without a prefix sum over the requests.
struct RowTile {
  int32_t s, row0, rows;  // rows <= 0: nothing to do
};
template <int SHIFT>
__device__ inline RowTile row_tile(const int32_t *q_off, int32_t n, int32_t b) {
  const int32_t lo =
      last_at_most(n, b, [&](int32_t s) { return (__ldg(q_off + s) >> SHIFT) + s; });
  const int32_t q0 = __ldg(q_off + lo), q1 = __ldg(q_off + lo + 1);
  RowTile t;
  t.s = lo;
  t.row0 = q0 + ((b - (q0 >> SHIFT) - lo) << SHIFT);
  t.rows = q1 - t.row0 < (1 << SHIFT) ? q1 - t.row0 : (1 << SHIFT);
  return t;
}
inline int64_t row_tiles(const fs_step *s, int shift) {
  return (int64_t(s->q_off_h[s->n_seqs]) >> shift) + s->n_seqs;
}

// A cache as kernels see it (page_size = 1 << page_shift).  Offsets are in elements; one
// inside a page fits 31 bits, as the page stride does (checked on the host).
struct DevCache {
  const char *k, *v;
  uint32_t page_stride, head_stride, token_stride, n_pages;
  const int32_t *table;
  int64_t table_stride;
  int32_t page_shift, n_kv_heads, head_dim;
};

inline DevCache dev_cache(const fs_kv_cache *c) {
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

// A request's cached length as a kernel may use it: checked against the host's bound
// (and so against the page table's width).  *code is raised for one outside.
__device__ inline int32_t checked_len(const int32_t *kv_len, int32_t s, int32_t max_kv,
                                      int32_t &code) {
  const int32_t n = __ldg(kv_len + s);
  if (n < 0 || n > max_kv) {
    code = FS_E_RANGE;
    return n < 0 ? 0 : max_kv;
  }
  return n;
}

// Offset of a token's row: its page (an id outside the cache raises *code and becomes page
// 0), its slot, and the head's offset inside a page.
__device__ inline uint64_t row_at(const DevCache &c, uint32_t page, int32_t j, uint32_t head,
                                  int32_t &code) {
  if (page >= c.n_pages) {
    code = FS_E_RANGE;
    page = 0;
  }
  return uint64_t(page) * c.page_stride +
         (head + uint32_t(j & ((1 << c.page_shift) - 1)) * c.token_stride);
}

// ---- launchers
size_t adapter_workspace_bytes(const fs_step *s, const fs_adapters *ad);
hipError_t launch_adapter_linear(const fs_step *s, const fs_adapters *ad, const void *x,
                                 int64_t x_stride, const void *w, void *y, int64_t y_stride,
                                 void *ws, int32_t *err, hipStream_t stream);

hipError_t launch_rope_append(const fs_step *s, const fs_kv_cache *c, const fs_rope *r,
                              int32_t n_heads, const void *q, int64_t q_stride, const void *k,
                              int64_t k_stride, const void *v, int64_t v_stride, void *q_out,
                              int64_t q_out_stride, int32_t *err, hipStream_t stream);

size_t attention_workspace_bytes(const fs_step *s, const fs_kv_cache *c, int32_t n_heads,
                                 int32_t window);
hipError_t launch_attention(const fs_step *s, const fs_kv_cache *c, int32_t n_heads, float scale,
                            int32_t window, const void *q, int64_t q_stride, void *out,
                            int64_t out_stride, float *lse, void *ws, int32_t *err,
                            hipStream_t stream);

size_t sample_workspace_bytes(int32_t dtype, int32_t rows, int32_t vocab);
hipError_t launch_sample(int32_t dtype, int32_t rows, int32_t vocab, const void *logits,
                         int64_t stride, const fs_sampling *p, const float *u, int32_t *token,
                         float *logprob, int32_t *kept, void *ws, int32_t *err,
                         hipStream_t stream);

}  // namespace fs
