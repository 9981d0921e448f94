// Rotary positions of the step's queries and keys, and the append of its keys and values
// to the paged cache, in one pass:
//   (a, b) -> (a cos t - b sin t, b cos t + a sin t) * factor,  t = p * inv_freq[i].
// The angle is reduced in fp64 (p reaches 2^24 and more: in fp32 its error would pass a
// bfloat16 ulp from p = 2^16 on), each cos and sin is computed once for all heads of a
// token, everything else is fp32 and is rounded once.  Bound by its bytes, each read and
// written once (5,700 rows of 32 + 2 x 8 heads of 128: 140 MB in 30.5 us, 4.6 TB/s), and at
// a few rows by the chain of lengths, page id, loads and stores (8 rows: 6.5 us).  Four
// tokens a work-group, so that 5,700 rows fill the card five times over and a decode step of
// 256 still has 64 work-groups.
#include "fs_engine.h"

namespace fs {

namespace {

struct RopeArgs {
  const int32_t *q_off, *kv_len;
  int32_t n_seqs, max_kv, rows;
  DevCache c;
  char *kw, *vw;  // the cache, for writing
  const char *q, *k, *v;
  char *q_out;
  int64_t q_stride, k_stride, v_stride, q_out_stride;
  const float *inv_freq;
  const int32_t *pos;
  float factor;
  int32_t n_heads, rotary;
  int32_t *err;
};

constexpr int kTok = 4;  // tokens per work-group

// Turns 8 elements a against 8 elements b (pairs (a[i], b[i])).
template <bool BF>
__device__ inline void turn8(s16x8 &a, s16x8 &b, const float *cs, const float *sn) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = to_f32<BF>(a[i]), y = to_f32<BF>(b[i]);
    a[i] = to_16<BF>(x * cs[i] - y * sn[i]);
    b[i] = to_16<BF>(y * cs[i] + x * sn[i]);
  }
}

// VEC: pairs lie in whole 16-byte chunks (rotary_dim a multiple of 16, or of 8 when
// interleaved); else one pair or one element per item.
template <bool BF, bool INTER, bool VEC>
__global__ void __launch_bounds__(256) k_rope_append(RopeArgs a) {
  __shared__ float cs[kTok][128], sn[kTok][128];
  __shared__ int64_t slot[kTok];  // the token's cache row (head 0), in elements; -1: none
  __shared__ int32_t where[kTok];
  const int32_t t0 = blockIdx.x * kTok;
  const int32_t nt = min(kTok, a.rows - t0);
  const int tid = threadIdx.x;
  // a wave for each token
  if (tid >> 6 < nt) {
    const int32_t i = tid >> 6, t = t0 + i;
    const int32_t s = seq_of_row(a.q_off, a.n_seqs, t);
    if ((tid & 63) == 0) {
      int32_t code = 0;
      const int32_t kv = checked_len(a.kv_len, s, a.max_kv, code);
      const int32_t p = kv - (__ldg(a.q_off + s + 1) - t);
      int64_t at = -1;
      if (p >= 0 && !code) {  // a length that is none says nothing of a token's place
        const uint32_t id = __ldg(a.c.table + s * a.c.table_stride + (p >> a.c.page_shift));
        if (id < a.c.n_pages)
          at = row_at(a.c, id, p, 0, code);
        else
          code = FS_E_RANGE;
      }
      slot[i] = at;
      where[i] = a.pos ? __ldg(a.pos + t) : max(p, 0);
      raise_err(a.err, code);
    }
  }
  __syncthreads();
  const int half = a.rotary / 2;
  for (int i = tid; i < nt * half; i += 256) {
    const int tok = i / half, f = i - tok * half;
    const double th = double(where[tok]) * double(__ldg(a.inv_freq + f));
    const double turns = th * 0.15915494309189533577;  // 1 / 2 pi
    const float r = float((turns - rint(turns)) * 6.283185307179586476925);
    float sv, cv;
    sincosf(r, &sv, &cv);
    cs[tok][f] = cv * a.factor;
    sn[tok][f] = sv * a.factor;
  }
  __syncthreads();

  const int D = a.c.head_dim, HK = a.c.n_kv_heads;
  // items of a head that turns, and of one that is copied
  const int turned = VEC ? (INTER ? a.rotary / 8 : a.rotary / 16) : half;
  const int rest = VEC ? (D - a.rotary) / 8 : D - a.rotary;
  const int per = turned + rest, vper = VEC ? D / 8 : D;
  const int rot_items = (a.n_heads + HK) * per;
  const int items = rot_items + HK * vper;
  for (int tok = 0; tok < nt; ++tok) {
    const int64_t t = t0 + tok;
    const int64_t at = slot[tok];
    for (int it = tid; it < items; it += 256) {
      const char *src;
      char *dst;
      int j;
      bool copy = false;
      if (it < rot_items) {
        const int h = it / per;
        j = it - h * per;
        if (h < a.n_heads) {
          src = a.q + 2 * (t * a.q_stride + h * D);
          dst = a.q_out + 2 * (t * a.q_out_stride + h * D);
        } else {
          if (at < 0) continue;
          src = a.k + 2 * (t * a.k_stride + (h - a.n_heads) * D);
          dst = a.kw + 2 * (at + int64_t(h - a.n_heads) * a.c.head_stride);
        }
      } else {
        if (at < 0) continue;
        const int r = it - rot_items, h = r / vper;
        j = r - h * vper;
        src = a.v + 2 * (t * a.v_stride + h * D);
        dst = a.vw + 2 * (at + int64_t(h) * a.c.head_stride);
        copy = true;
      }
      if constexpr (VEC) {
        if (copy || j >= turned) {
          const int e = copy ? j * 8 : a.rotary + (j - turned) * 8;
          *reinterpret_cast<s16x8 *>(dst + 2 * e) = *reinterpret_cast<const s16x8 *>(src + 2 * e);
        } else if constexpr (INTER) {
          s16x8 x = *reinterpret_cast<const s16x8 *>(src + 16 * j);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float c = cs[tok][4 * j + i], sv = sn[tok][4 * j + i];
            const float p = to_f32<BF>(x[2 * i]), q = to_f32<BF>(x[2 * i + 1]);
            x[2 * i] = to_16<BF>(p * c - q * sv);
            x[2 * i + 1] = to_16<BF>(q * c + p * sv);
          }
          *reinterpret_cast<s16x8 *>(dst + 16 * j) = x;
        } else {
          s16x8 x = *reinterpret_cast<const s16x8 *>(src + 16 * j);
          s16x8 y = *reinterpret_cast<const s16x8 *>(src + 16 * j + a.rotary);
          turn8<BF>(x, y, &cs[tok][8 * j], &sn[tok][8 * j]);
          *reinterpret_cast<s16x8 *>(dst + 16 * j) = x;
          *reinterpret_cast<s16x8 *>(dst + 16 * j + a.rotary) = y;
        }
      } else {
        const short *sp = reinterpret_cast<const short *>(src);
        short *dp = reinterpret_cast<short *>(dst);
        if (copy || j >= turned) {
          const int e = copy ? j : a.rotary + j - turned;
          dp[e] = sp[e];
        } else {
          const int e0 = INTER ? 2 * j : j, e1 = INTER ? 2 * j + 1 : j + half;
          const float p = to_f32<BF>(sp[e0]), q = to_f32<BF>(sp[e1]);
          dp[e0] = to_16<BF>(p * cs[tok][j] - q * sn[tok][j]);
          dp[e1] = to_16<BF>(q * cs[tok][j] + p * sn[tok][j]);
        }
      }
    }
  }
}

template <bool BF>
void run(const RopeArgs &a, bool inter, bool vec, hipStream_t stream) {
  const dim3 grid((a.rows + kTok - 1) / kTok), block(256);
  if (inter && vec)
    hipLaunchKernelGGL((k_rope_append<BF, true, true>), grid, block, 0, stream, a);
  else if (inter)
    hipLaunchKernelGGL((k_rope_append<BF, true, false>), grid, block, 0, stream, a);
  else if (vec)
    hipLaunchKernelGGL((k_rope_append<BF, false, true>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((k_rope_append<BF, false, false>), grid, block, 0, stream, a);
}

}  // namespace

hipError_t launch_rope_append(const fs_step *s, const fs_kv_cache *c, const fs_rope *r,
                              int32_t n_heads, const void *q, int64_t q_stride, const void *k,
                              int64_t k_stride, const void *v, int64_t v_stride, void *q_out,
                              int64_t q_out_stride, int32_t *err, hipStream_t stream) {
  RopeArgs a;
  a.q_off = s->q_off;
  a.kv_len = s->kv_len;
  a.n_seqs = s->n_seqs;
  a.max_kv = s->max_kv;
  a.rows = s->q_off_h[s->n_seqs];
  a.c = dev_cache(c);
  a.kw = static_cast<char *>(c->k);
  a.vw = static_cast<char *>(c->v);
  a.q = static_cast<const char *>(q);
  a.k = static_cast<const char *>(k);
  a.v = static_cast<const char *>(v);
  a.q_out = static_cast<char *>(q_out);
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_out_stride = q_out_stride;
  a.inv_freq = r->inv_freq;
  a.pos = r->pos;
  a.factor = r->factor;
  a.n_heads = n_heads;
  a.rotary = r->rotary_dim;
  a.err = err;
  const bool inter = r->interleaved != 0;
  const bool vec = r->rotary_dim % (inter ? 8 : 16) == 0;
  if (c->dtype == FS_BF16)
    run<true>(a, inter, vec, stream);
  else
    run<false>(a, inter, vec, stream);
  return hipGetLastError();
}

}  // namespace fs
