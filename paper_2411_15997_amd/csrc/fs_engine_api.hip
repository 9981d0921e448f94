// extern "C" entry points of the engine-step operators (declared in
// include/fairserve_engine.h): synchronous argument checks, then the launchers.
#include <cmath>

#include "fs_check.h"
#include "fs_launch.h"

namespace fs {
namespace {

fs_status check_adapters(const fs_adapters *ad) {
  if (!ad || (ad->dtype != FS_BF16 && ad->dtype != FS_F16)) return FS_E_ARG;
  if (ad->in_features < 8 || ad->out_features < 8 || !mult8(ad->in_features) ||
      !mult8(ad->out_features) || ad->in_features > (1 << 20) || ad->out_features > (1 << 20))
    return FS_E_ARG;
  if (ad->n_adapters < 0) return FS_E_ARG;
  if (ad->n_adapters > 0) {
    if (ad->max_rank < 8 || ad->max_rank > 128 || !mult8(ad->max_rank)) return FS_E_ARG;
    if (!ad->a || !ad->b || !ad->adapter || !aligned_to(ad->a, 16) || !aligned_to(ad->b, 16))
      return FS_E_ARG;
  }
  return FS_OK;
}

}  // namespace
}  // namespace fs

using namespace fs;

extern "C" {

fs_status fs_clear_status(int32_t *err, hipStream_t stream) {
  if (!err) return FS_E_ARG;
  return status_of(launch_zero_i32(err, stream));
}

size_t fs_adapter_workspace(const fs_step *s, const fs_adapters *ad) {
  if (check_step(s, false) != FS_OK || check_adapters(ad) != FS_OK) return 0;
  return adapter_workspace_bytes(s, ad);
}

fs_status fs_adapter_linear(const fs_step *s, const fs_adapters *ad, const void *x,
                            int64_t x_stride, const void *w, void *y, int64_t y_stride, void *ws,
                            size_t ws_bytes, int32_t *err, hipStream_t stream) {
  fs_status st = check_step(s, false);
  if (st == FS_OK) st = check_adapters(ad);
  if (st != FS_OK) return st;
  if (!err) return FS_E_ARG;
  if (rows_of(s) == 0) return FS_OK;
  if (!x || !w || !y || !aligned_to(x, 16) || !aligned_to(w, 16) || !aligned_to(y, 16) ||
      !mult8(x_stride) || !mult8(y_stride) || x_stride < ad->in_features ||
      y_stride < ad->out_features || x_stride > (1 << 21))
    return FS_E_ARG;
  const size_t need = adapter_workspace_bytes(s, ad);
  if (need > 0 && (!ws || !aligned_to(ws, 256) || ws_bytes < need)) return FS_E_WORKSPACE;
  return status_of(launch_adapter_linear(s, ad, x, x_stride, w, y, y_stride, ws, err, stream));
}

fs_status fs_rope_frequencies(int32_t rotary_dim, double theta0, int32_t scaling, double scale,
                              int32_t original_len, double beta_fast, double beta_slow,
                              float *inv_freq_h, float *factor_h) {
  if (rotary_dim < 0 || rotary_dim > 256 || (rotary_dim & 1) || !(theta0 > 0.0) ||
      !std::isfinite(theta0) || scaling < FS_ROPE_PLAIN || scaling > FS_ROPE_PARTS || !factor_h ||
      (rotary_dim > 0 && !inv_freq_h))
    return FS_E_ARG;
  if (scaling != FS_ROPE_PLAIN && (!(scale >= 1.0) || !std::isfinite(scale))) return FS_E_ARG;
  if (scaling == FS_ROPE_BASE && rotary_dim == 2) return FS_E_ARG;
  if (scaling == FS_ROPE_PARTS &&
      (original_len < 1 || !(beta_fast > beta_slow) || !std::isfinite(beta_fast) ||
       !std::isfinite(beta_slow)))
    return FS_E_ARG;
  const double kTwoPi = 6.283185307179586476925287;
  double base = theta0;
  if (scaling == FS_ROPE_BASE)
    base = theta0 * std::pow(scale, double(rotary_dim) / (rotary_dim - 2));
  for (int32_t i = 0; i < rotary_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rotary_dim);
    if (scaling == FS_ROPE_LINEAR) f /= scale;
    if (scaling == FS_ROPE_PARTS) {
      const double turns = original_len * f / kTwoPi;
      double keep = (turns - beta_slow) / (beta_fast - beta_slow);
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
      f = f / scale * (1.0 - keep) + f * keep;
    }
    inv_freq_h[i] = float(f);
  }
  *factor_h = scaling == FS_ROPE_PARTS ? float(0.1 * std::log(scale) + 1.0) : 1.0f;
  return FS_OK;
}

fs_status fs_rope_append(const fs_step *s, const fs_kv_cache *c, const fs_rope *r,
                         int32_t n_heads, const void *q, int64_t q_stride, const void *k,
                         int64_t k_stride, const void *v, int64_t v_stride, void *q_out,
                         int64_t q_out_stride, int32_t *err, hipStream_t stream) {
  fs_status st = check_step(s, true);
  if (st == FS_OK) st = check_cache(s, c, 256);
  if (st != FS_OK) return st;
  if (!r || !err || r->rotary_dim < 0 || r->rotary_dim > c->head_dim || (r->rotary_dim & 1) ||
      r->interleaved < 0 || r->interleaved > 1 || (r->rotary_dim > 0 && !r->inv_freq) ||
      n_heads < 0 || n_heads > 65535)
    return FS_E_ARG;
  if (rows_of(s) == 0) return FS_OK;
  const int64_t row = int64_t(c->n_kv_heads) * c->head_dim;
  if (!k || !v || !aligned_to(k, 16) || !aligned_to(v, 16) || !mult8(k_stride) ||
      !mult8(v_stride) || k_stride < row || v_stride < row)
    return FS_E_ARG;
  if (n_heads > 0) {
    const int64_t qrow = int64_t(n_heads) * c->head_dim;
    if (!q || !q_out || !aligned_to(q, 16) || !aligned_to(q_out, 16) || !mult8(q_stride) ||
        !mult8(q_out_stride) || q_stride < qrow || q_out_stride < qrow)
      return FS_E_ARG;
  }
  return status_of(launch_rope_append(s, c, r, n_heads, q, q_stride, k, k_stride, v, v_stride,
                                      q_out, q_out_stride, err, stream));
}

size_t fs_attention_workspace(const fs_step *s, const fs_kv_cache *c, int32_t n_heads,
                              int32_t window) {
  if (check_attention(s, c, n_heads, window, 0) != FS_OK) return 0;
  return attention_workspace_bytes(s, c, n_heads, window, 0);
}

fs_status fs_paged_attention(const fs_step *s, const fs_kv_cache *c, int32_t n_heads, float scale,
                             int32_t window, const void *q, int64_t q_stride, void *out,
                             int64_t out_stride, float *lse, void *ws, size_t ws_bytes,
                             int32_t *err, hipStream_t stream) {
  fs_status st = check_attention(s, c, n_heads, window, 0);
  if (st != FS_OK) return st;
  if (!err || !std::isfinite(scale)) return FS_E_ARG;
  if (rows_of(s) == 0) return FS_OK;
  const int64_t row = int64_t(n_heads) * c->head_dim;
  if (!q || !out || !aligned_to(q, 16) || !aligned_to(out, 16) || !mult8(q_stride) ||
      !mult8(out_stride) || q_stride < row || out_stride < row)
    return FS_E_ARG;
  const size_t need = attention_workspace_bytes(s, c, n_heads, window, 0);
  if (need > 0 && (!ws || !aligned_to(ws, 256) || ws_bytes < need)) return FS_E_WORKSPACE;
  return status_of(launch_attention(s, c, n_heads, scale, window, 0, q, q_stride, out, out_stride,
                                    lse, ws, err, stream));
}

size_t fs_sample_workspace(int32_t dtype, int32_t rows, int32_t vocab) {
  if (dtype < FS_BF16 || dtype > FS_F32 || rows < 0 || vocab < 1 || vocab > (1 << 20)) return 0;
  return sample_workspace_bytes(dtype, rows, vocab);
}

fs_status fs_sample(int32_t dtype, int32_t rows, int32_t vocab, const void *logits, int64_t stride,
                    const fs_sampling *p, const float *u, int32_t *token, float *logprob,
                    int32_t *kept, void *ws, size_t ws_bytes, int32_t *err, hipStream_t stream) {
  if (dtype < FS_BF16 || dtype > FS_F32 || rows < 0 || rows > (1 << 21) || vocab < 1 ||
      vocab > (1 << 20) || !p || !err || stride < vocab)
    return FS_E_ARG;
  if (rows == 0) return FS_OK;
  if (!logits || !u || !token || !aligned_to(logits, dtype == FS_F32 ? 4 : 2)) return FS_E_ARG;
  const size_t need = sample_workspace_bytes(dtype, rows, vocab);
  if (need > 0 && (!ws || !aligned_to(ws, 256) || ws_bytes < need)) return FS_E_WORKSPACE;
  return status_of(launch_sample(dtype, rows, vocab, logits, stride, p, u, token, logprob, kept,
                                 ws, err, stream));
}

}  // extern "C"
