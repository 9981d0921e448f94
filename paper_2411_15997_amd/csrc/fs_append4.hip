// Rotary positions of the step's queries and keys, and the append of its keys and values to
// a cache held in 4 bits; and the step's rows of such a cache, read back.
//
//   (a, b) -> (a cos t - b sin t, b cos t + a sin t) * factor,  t = p * inv_freq[i];
//   a group x of 32 values: E least with max |x| <= 7 * 2^E, codes of x / 2^E.
// Keys are turned in fp64 (the angle, its sine and cosine, the products) and rounded to fp32
// once: next to the border of two codes an error of fp32 would pick the other one, half of the
// value away, and the cache would hang on the order of operations.  A key value costs two
// fp64 products, which the card does at half of its fp32 rate.
// Bound by HBM in steps of thousands of rows (7,616 of 32 + 2 x 8 heads of 128: 30 us, 5.4 TB/s,
// and 9, 4.4 TB/s, to read them back), by the chain from lengths to pages to rows in small ones
// (8 rows: 5.0 us and 3.2).
#include <type_traits>

#include "fs_cache.h"

namespace fs {

namespace {

struct Append4Args {
  const int32_t *q_off, *kv_len;
  int32_t n_seqs, max_kv, rows;
  DevCache c;
  DevScales sc;
  char *kw, *vw;  // the codes, for writing
  uint8_t *ksw, *vsw;
  const short *q, *k, *v;
  short *q_out, *k_out, *v_out;
  int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride, v_out_stride;
  const float *inv_freq;
  const int32_t *pos;
  float factor;
  int32_t n_heads, rotary;
  int32_t *err;
};

// A token's place: its cache rows of head 0 (bytes; -1: none) and its position.
struct Place {
  int64_t code, scale;
  int32_t pos;
};
// Of row t, by the whole wave.
__device__ inline Place place_of(const Append4Args &a, int32_t t, int32_t &code) {
  const int32_t s = seq_of_row(a.q_off, a.n_seqs, t);
  const int32_t kv = checked_len(a.kv_len, s, a.max_kv, code);
  const int32_t p = kv - (__ldg(a.q_off + s + 1) - t);
  Place w = {-1, -1, p};
  if (p >= 0 && !code) {  // a length that is none says nothing of a token's place
    const uint32_t id = __ldg(a.c.table + s * a.c.table_stride + (p >> a.c.page_shift));
    if (id < a.c.n_pages) {
      const uint32_t slot = uint32_t(p & ((1 << a.c.page_shift) - 1));
      w.code = int64_t(id) * a.c.page_stride + int64_t(slot) * a.c.token_stride;
      w.scale = int64_t(id) * a.sc.page_stride + int64_t(slot) * a.sc.token_stride;
    } else {
      code = FS_E_RANGE;
    }
  }
  return w;
}

// Eight of a group's values, the others with the next three lanes: their codes, and the group's
// scale byte.
template <bool BF>
__device__ inline uint32_t codes8(const float *x, uint32_t &byte) {
  uint32_t top = 0;  // of the absolute values' bits: what is not finite is above all others
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = max(top, uint32_t(__shfl_xor(int(top), 1, 64)));
  top = max(top, uint32_t(__shfl_xor(int(top), 2, 64)));
  if (top >= 0x7f800000u) {
    byte = 255;
    return 0;
  }
  // top = f 2^e <= 7 * 2^E = 1.75 * 2^(E + 2)
  const int32_t e = int32_t(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  byte = uint32_t(min(max(e, 1), int32_t(kTopScale<BF>)));
  const float unit = __uint_as_float(byte << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], unit, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], unit, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], unit, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], unit, 3);
  return w;
}

// Element d of a row turned in F: x with the other element of its pair.
template <class F, bool INTER>
__device__ inline float turned(int d, int half, float x, float other, const F *cs, const F *sn) {
  const int f = INTER ? d >> 1 : d < half ? d : d - half;
  const bool second = INTER ? d & 1 : d >= half;
  return float(second ? F(x) * cs[f] + F(other) * sn[f] : F(x) * cs[f] - F(other) * sn[f]);
}

// A key's chunk of 8 elements is turned by one lane, which reads the pairs' other elements too;
// queries may be turned in place, so there a lane takes both.  Without INTER these lie half of
// rotary_dim apart, and PW of them (8, 4 or 1, which divides that) are one load; with INTER PW is
// 8 where whole chunks are turned.  (6,629 rows of 32 + 2 x 8 heads, 24 of 128 elements turned,
// and the rows read back: 45.6 us, 102.6 by single elements; 6,916 rows and 22 elements 82, 40.7
// interleaved.)
// TOK tokens a work-group.
template <bool BF, bool INTER, int PW, int TOK>
__global__ void __launch_bounds__(256) k_rope_append4(Append4Args a) {
  typedef short __attribute__((ext_vector_type(PW))) Side;  // one side of the pairs of a lane
  __shared__ double cs[TOK][128], sn[TOK][128];
  __shared__ float csf[TOK][128], snf[TOK][128];  // rounded, for the queries
  __shared__ Place place[TOK];
  const int32_t t0 = blockIdx.x * TOK;
  const int32_t nt = min(TOK, a.rows - t0);
  const int tid = threadIdx.x;
  // a wave for each token
  if (tid >> 6 < nt) {
    const int32_t i = tid >> 6, t = t0 + i;
    int32_t code = 0;
    Place w = place_of(a, t, code);
    if ((tid & 63) == 0) {
      w.pos = a.pos ? __ldg(a.pos + t) : max(w.pos, 0);
      place[i] = w;
      raise_err(a.err, code);
    }
  }
  __syncthreads();
  const int half = a.rotary / 2, D = a.c.head_dim, HK = a.c.n_kv_heads;
  for (int i = tid; i < nt * half; i += 256) {
    const int tok = i / half, f = i - tok * half;
    double sv, cv;
    sincos(double(place[tok].pos) * double(__ldg(a.inv_freq + f)), &sv, &cv);
    cv *= double(a.factor), sv *= double(a.factor);
    cs[tok][f] = cv, sn[tok][f] = sv;
    csf[tok][f] = float(cv), snf[tok][f] = float(sv);
  }
  __syncthreads();

  const int CH = D / 8;  // 8-element chunks of a head
  const int kv_items = HK * CH;
  // A thread has the same item of all the work-group's tokens under way: one look for its place
  // in the row, and TOK loads before the first is waited for.  (7,616 rows of
  // 32 + 2 x 8 heads: 31.5 us, 36 with one item after the other.)
  for (int it = tid; it < 2 * kv_items; it += 256) {
    const bool val = it >= kv_items;
    const int r = val ? it - kv_items : it, h = r / CH, ch = r - h * CH;
    const int64_t stride = val ? a.v_stride : a.k_stride;
    const short *row = (val ? a.v : a.k) + t0 * stride + h * D;
    const bool turn = !val && ch * 8 < a.rotary;
    s16x8 in[TOK];
    Side other[TOK][8 / PW];
#pragma unroll
    for (int u = 0; u < TOK; ++u) {
      const short *from = row + min(u, nt - 1) * stride;
      in[u] = *reinterpret_cast<const s16x8 *>(from + ch * 8);
      if (!INTER && PW > 1 && turn)  // the pairs' other elements
#pragma unroll
        for (int g = 0; g < 8 / PW; ++g) {
          const int d = ch * 8 + g * PW;
          other[u][g] = *reinterpret_cast<const Side *>(from + (d < half ? d + half : d - half));
        }
    }
#pragma unroll
    for (int u = 0; u < TOK; ++u) {
      if (u >= nt) break;
      const Place at = place[u];
      if (at.code < 0) continue;
      const double *c = cs[u], *s = sn[u];
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = to_f32<BF>(in[u][i]);
      if (turn) {
        if constexpr (INTER) {
#pragma unroll
          for (int i = 0; i < 8; i += 2)
            if (PW == 8 || ch * 8 + i < a.rotary) {
              const float p = x[i], q = x[i + 1];
              x[i] = turned<double, INTER>(ch * 8 + i, half, p, q, c, s);
              x[i + 1] = turned<double, INTER>(ch * 8 + i + 1, half, q, p, c, s);
            }
        } else if constexpr (PW > 1) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            x[i] = turned<double, INTER>(ch * 8 + i, half, x[i],
                                         to_f32<BF>(other[u][i / PW][i % PW]), c, s);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int d = ch * 8 + i;
            if (d < a.rotary)
              x[i] = turned<double, INTER>(
                  d, half, x[i], to_f32<BF>(row[u * stride + (d < half ? d + half : d - half)]), c,
                  s);
          }
        }
      }
      uint32_t byte;  // (a group is four neighbouring lanes': CH is a multiple of 4)
      const uint32_t w = codes8<BF>(x, byte);
      *reinterpret_cast<uint32_t *>((val ? a.vw : a.kw) + at.code + int64_t(h) * a.c.head_stride +
                                    ch * 4) = w;
      if ((ch & 3) == 0)
        ((val ? a.vsw : a.ksw) + at.scale + int64_t(h) * a.sc.head_stride)[ch >> 2] = uint8_t(byte);
    }
  }

  // of a head's items: turned ones, single elements up to a whole chunk, chunks that stay
  const int q_turned = INTER ? (a.rotary + 7) / 8 : half / PW;
  const int edge = !INTER && PW == 1 ? -a.rotary & 7 : 0, rest = (a.rotary + 7) & ~7;
  const int per = q_turned + edge + (D - rest) / 8;
  for (int it = tid; it < a.n_heads * per; it += 256) {
    const int h = it / per, j = it - h * per;
    const bool turn = j < q_turned;
    const short *src = a.q + t0 * a.q_stride + h * D;
    short *dst = a.q_out + t0 * a.q_out_stride + h * D;
    if (edge && !turn && j < q_turned + edge) {
      const int e = a.rotary + j - q_turned;
      for (int u = 0; u < nt; ++u) dst[u * a.q_out_stride + e] = src[u * a.q_stride + e];
      continue;
    }
    const int e = turn ? (INTER ? 8 : PW) * j : rest + (j - q_turned - edge) * 8;
    src += e, dst += e;
    s16x8 in[TOK];
    Side other[TOK];
#pragma unroll
    for (int u = 0; u < TOK; ++u) {
      const short *from = src + min(u, nt - 1) * a.q_stride;
      if (INTER || PW == 8 || !turn) {
        in[u] = *reinterpret_cast<const s16x8 *>(from);
      } else {
        const Side x = *reinterpret_cast<const Side *>(from);
#pragma unroll
        for (int i = 0; i < PW; ++i) in[u][i] = x[i];
      }
      if (!INTER && turn) other[u] = *reinterpret_cast<const Side *>(from + half);
    }
#pragma unroll
    for (int u = 0; u < TOK; ++u) {
      if (u >= nt) break;
      const float *c = csf[u], *s = snf[u];
      short *to = dst + u * a.q_out_stride;
      s16x8 v = in[u];
      if (INTER && turn) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (PW == 8 || e + i < a.rotary)
            v[i] = to_16<BF>(turned<float, INTER>(e + i, half, to_f32<BF>(in[u][i]),
                                                  to_f32<BF>(in[u][i ^ 1]), c, s));
      } else if (turn) {
        Side w;
#pragma unroll
        for (int i = 0; i < PW; ++i) {
          const float p = to_f32<BF>(in[u][i]), q = to_f32<BF>(other[u][i]);
          v[i] = to_16<BF>(turned<float, INTER>(e + i, half, p, q, c, s));
          w[i] = to_16<BF>(turned<float, INTER>(e + i + half, half, q, p, c, s));
        }
        *reinterpret_cast<Side *>(to + half) = w;
        if constexpr (PW < 8) {
          Side x;
#pragma unroll
          for (int i = 0; i < PW; ++i) x[i] = v[i];
          *reinterpret_cast<Side *>(to) = x;
          continue;
        }
      }
      *reinterpret_cast<s16x8 *>(to) = v;
    }
  }
}

// What the cache holds at the step's rows.
template <bool BF, int TOK>
__global__ void __launch_bounds__(256) k_cache4_rows(Append4Args a) {
  __shared__ Place place[TOK];
  const int32_t t0 = blockIdx.x * TOK;
  const int32_t nt = min(TOK, a.rows - t0);
  const int tid = threadIdx.x;
  if (tid >> 6 < nt) {
    int32_t code = 0;
    const Place w = place_of(a, t0 + (tid >> 6), code);
    if ((tid & 63) == 0) {
      place[tid >> 6] = w;
      raise_err(a.err, code);
    }
  }
  __syncthreads();
  const int D = a.c.head_dim, CH = D / 8, kv_items = a.c.n_kv_heads * CH;
  for (int it = tid; it < 2 * kv_items; it += 256) {
    const bool val = it >= kv_items;
    const int r = val ? it - kv_items : it, h = r / CH, ch = r - h * CH;
    const int64_t stride = val ? a.v_out_stride : a.k_out_stride;
    short *out = val ? a.v_out : a.k_out;
    if (!out) continue;
    out += t0 * stride + h * D + ch * 8;
    uint32_t w[TOK], byte[TOK];
#pragma unroll
    for (int u = 0; u < TOK; ++u) {
      const Place at = place[min(u, nt - 1)];
      w[u] = byte[u] = 0;
      if (at.code < 0) continue;
      w[u] = *reinterpret_cast<const uint32_t *>((val ? a.c.v : a.c.k) + at.code +
                                                 int64_t(h) * a.c.head_stride + ch * 4);
      byte[u] = ((val ? a.sc.v : a.sc.k) + at.scale + int64_t(h) * a.sc.head_stride)[ch >> 2];
    }
#pragma unroll
    for (int u = 0; u < TOK; ++u) {
      if (u >= nt) break;
      s16x8 x = values8<BF>(w[u], scale_of<BF>(byte[u]));
      if (byte[u] > kTopScale<BF>) x = BF ? 0x7fc0 : 0x7e00;  // NaN
      *reinterpret_cast<s16x8 *>(out + u * stride) = x;
    }
  }
}

// One token a work-group up to 1,024 rows, where a work-group's items would only follow each
// other (8 rows: 5.0 us, 10.4 with four), and four beyond, which look for their places side by side.
template <class F>
void by_rows(int32_t rows, int32_t dtype, F f) {
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 4> four;
  if (dtype == FS_BF16)
    rows <= 1024 ? f(std::true_type(), one) : f(std::true_type(), four);
  else
    rows <= 1024 ? f(std::false_type(), one) : f(std::false_type(), four);
}

Append4Args step_args(const fs_step *s, const fs_kv_cache4 *c, int32_t *err) {
  Append4Args a = {};
  a.q_off = s->q_off;
  a.kv_len = s->kv_len;
  a.n_seqs = s->n_seqs;
  a.max_kv = s->max_kv;
  a.rows = s->q_off_h[s->n_seqs];
  a.c = dev_codes(c);
  a.sc = dev_scales(c);
  a.kw = static_cast<char *>(c->k);
  a.vw = static_cast<char *>(c->v);
  a.ksw = static_cast<uint8_t *>(c->k_scale);
  a.vsw = static_cast<uint8_t *>(c->v_scale);
  a.err = err;
  return a;
}

}  // namespace

hipError_t launch_rope_append4(const fs_step *s, const fs_kv_cache4 *c, const fs_rope *r,
                               int32_t dtype, int32_t n_heads, const void *q, int64_t q_stride,
                               const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                               void *q_out, int64_t q_out_stride, int32_t *err,
                               hipStream_t stream) {
  Append4Args a = step_args(s, c, err);
  a.q = static_cast<const short *>(q);
  a.k = static_cast<const short *>(k);
  a.v = static_cast<const short *>(v);
  a.q_out = static_cast<short *>(q_out);
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_out_stride = q_out_stride;
  a.inv_freq = r->inv_freq;
  a.pos = r->pos;
  a.factor = r->factor;
  a.n_heads = n_heads;
  a.rotary = r->rotary_dim;
  const int half = r->rotary_dim / 2;
  by_rows(a.rows, dtype, [&](auto bf, auto tok) {
    constexpr bool BF = decltype(bf)::value;
    constexpr int TOK = decltype(tok)::value;
    const dim3 grid((a.rows + TOK - 1) / TOK), block(256);
    if (r->interleaved && r->rotary_dim % 8 == 0)
      hipLaunchKernelGGL((k_rope_append4<BF, true, 8, TOK>), grid, block, 0, stream, a);
    else if (r->interleaved)
      hipLaunchKernelGGL((k_rope_append4<BF, true, 1, TOK>), grid, block, 0, stream, a);
    else if (half % 8 == 0)
      hipLaunchKernelGGL((k_rope_append4<BF, false, 8, TOK>), grid, block, 0, stream, a);
    else if (half % 4 == 0)
      hipLaunchKernelGGL((k_rope_append4<BF, false, 4, TOK>), grid, block, 0, stream, a);
    else
      hipLaunchKernelGGL((k_rope_append4<BF, false, 1, TOK>), grid, block, 0, stream, a);
  });
  return hipGetLastError();
}

hipError_t launch_cache4_rows(const fs_step *s, const fs_kv_cache4 *c, int32_t dtype, void *k_out,
                              int64_t k_stride, void *v_out, int64_t v_stride, int32_t *err,
                              hipStream_t stream) {
  Append4Args a = step_args(s, c, err);
  a.k_out = static_cast<short *>(k_out);
  a.v_out = static_cast<short *>(v_out);
  a.k_out_stride = k_stride;
  a.v_out_stride = v_stride;
  by_rows(a.rows, dtype, [&](auto bf, auto tok) {
    constexpr int TOK = decltype(tok)::value;
    hipLaunchKernelGGL((k_cache4_rows<decltype(bf)::value, TOK>), dim3((a.rows + TOK - 1) / TOK),
                       dim3(256), 0, stream, a);
  });
  return hipGetLastError();
}

}  // namespace fs
