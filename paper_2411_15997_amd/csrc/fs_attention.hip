// Attention of the step's rows over the paged cache (one pass over the keys with the
// running maximum and sum of the softmax).  One wave per row and head.
#include "fs_engine.h"

namespace fs {

namespace {

struct AttnArgs {
  const int32_t *q_off, *kv_len;
  int32_t n_seqs, max_kv, rows, n_heads, window;
  DevCache c;
  const short *q;
  short *out;
  int64_t q_stride, out_stride;
  float *lse;
  float scale;
  int32_t *err;
};

template <bool BF, int D>
__global__ void __launch_bounds__(256) k_attention(AttnArgs a) {
  __shared__ float qs[4][D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t rh = int64_t(blockIdx.x) * 4 + wave;
  const bool live = rh < int64_t(a.rows) * a.n_heads;
  const int32_t t = live ? int32_t(rh / a.n_heads) : 0, h = live ? int32_t(rh % a.n_heads) : 0;
  for (int d = lane; d < D; d += 64)
    qs[wave][d] = to_f32<BF>(a.q[t * a.q_stride + h * D + d]) * a.scale;
  __syncthreads();
  if (!live) return;
  int32_t code = 0;
  const int32_t s = seq_of_row(a.q_off, a.n_seqs, t);
  const int32_t kv = checked_len(a.kv_len, s, a.max_kv, code);
  const int32_t p = kv - (__ldg(a.q_off + s + 1) - t);
  const int32_t first = a.window ? max(0, p - a.window + 1) : 0;
  const int64_t head = (h / (a.n_heads / a.c.n_kv_heads)) * a.c.head_stride;
  const int32_t *table = a.c.table + s * a.c.table_stride;
  const int32_t in_page = (1 << a.c.page_shift) - 1;
  float m = -INFINITY, l = 0.f, o[D / 64] = {};
  for (int32_t j0 = first; j0 <= p; j0 += 64) {
    const int32_t j = j0 + lane;
    const bool see = j <= p;
    int64_t at = 0;
    float sc = -INFINITY;
    if (see) {
      at = checked_page(a.c, table + (j >> a.c.page_shift), code) * a.c.page_stride + head +
           (j & in_page) * a.c.token_stride;
      const short *kp = reinterpret_cast<const short *>(a.c.k) + at;
      sc = 0.f;
      for (int d = 0; d < D; d += 8) {
        const s16x8 kv8 = *reinterpret_cast<const s16x8 *>(kp + d);
#pragma unroll
        for (int i = 0; i < 8; ++i) sc += to_f32<BF>(kv8[i]) * qs[wave][d + i];
      }
    }
    float top = sc;
    for (int w = 32; w; w >>= 1) top = fmaxf(top, __shfl_xor(top, w, 64));
    const float m2 = fmaxf(m, top);
    if (m2 == -INFINITY) continue;
    const float f = expf(m - m2), e = expf(sc - m2);
    float sum = e;
    for (int w = 32; w; w >>= 1) sum += __shfl_xor(sum, w, 64);
    l = l * f + sum;
    m = m2;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) o[i] *= f;
    const int n = min(64, p - j0 + 1);
    for (int i = 0; i < n; ++i) {
      const float w = __shfl(e, i, 64);
      const int64_t vat = __shfl(at, i, 64);
      const short *vp = reinterpret_cast<const short *>(a.c.v) + vat;
#pragma unroll
      for (int d = 0; d < D / 64; ++d) o[d] += w * to_f32<BF>(vp[d * 64 + lane]);
    }
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int d = 0; d < D / 64; ++d)
    a.out[t * a.out_stride + h * D + d * 64 + lane] = to_16<BF>(o[d] * inv);
  if (a.lse && lane == 0) a.lse[int64_t(t) * a.n_heads + h] = m + logf(l);
  raise_err(a.err, code);
}

}  // namespace

size_t attention_workspace_bytes(const fs_step *, const fs_kv_cache *, int32_t, int32_t) {
  return 0;
}

hipError_t launch_attention(const fs_step *s, const fs_kv_cache *c, int32_t n_heads, float scale,
                            int32_t window, const void *q, int64_t q_stride, void *out,
                            int64_t out_stride, float *lse, void *ws, int32_t *err,
                            hipStream_t stream) {
  AttnArgs a;
  a.q_off = s->q_off;
  a.kv_len = s->kv_len;
  a.n_seqs = s->n_seqs;
  a.max_kv = s->max_kv;
  a.rows = s->q_off_h[s->n_seqs];
  a.n_heads = n_heads;
  a.window = window;
  a.c = dev_cache(c);
  a.q = static_cast<const short *>(q);
  a.out = static_cast<short *>(out);
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.lse = lse;
  a.scale = scale;
  a.err = err;
  const dim3 grid((int64_t(a.rows) * n_heads + 3) / 4), block(256);
  const bool bf = c->dtype == FS_BF16;
  if (bf && c->head_dim == 128)
    hipLaunchKernelGGL((k_attention<true, 128>), grid, block, 0, stream, a);
  else if (bf)
    hipLaunchKernelGGL((k_attention<true, 64>), grid, block, 0, stream, a);
  else if (c->head_dim == 128)
    hipLaunchKernelGGL((k_attention<false, 128>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((k_attention<false, 64>), grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace fs
