// Attention of the step's rows over the paged cache: one pass over the keys with the
// running maximum and sum of the softmax.
//
// The G = n_heads / n_kv_heads query heads that share a key/value head are rows of one
// matrix product: a request's n tokens are n * G rows (token-major) per key/value head.
//   k_attn_few    requests of at most 64 rows (single tokens, small chunks): bound by the
//                 cache's bytes (64 requests of up to 16,384 tokens: 121 us, 4.97 TB/s; one of
//                 200,001: 80 us and 7 for the join, 5.1 TB/s).  The keys are spread over
//                 work-groups (splits of 512 to 1,024, more where their results would take too
//                 much memory; up to 131,072 / head_dim keys whole where the card has a unit
//                 for each request and head) and over the waves of each, which load 32 keys at
//                 a time into LDS of their own and never wait for each other.
//   k_attn_chunk  larger chunks: bound by the waits of a tile's chain (scores, maximum,
//                 exponentials, products) at two waves a SIMD; the matrix cores are busy for
//                 half of the cycles (4,096 rows over 32,768 keys, head_dim 128: 1.91 ms, 1.08
//                 PFLOP/s, 1.84 to 2.04 ms from card to card; head_dim 64: 0.84 PFLOP/s).  128 or
//                 256 rows a work-group share each tile of 64 keys.
//   k_attn_join_* join the splits' results with their maxima and sums, in split order.
// Both products run with the keys as rows of the first operand (S^T = K Q^T,
// O^T = V^T P^T): a lane then holds scores of one query row only, its probabilities are
// the second product's operand as they lie in registers, and the running factors are one
// number per lane.  The second product takes the keys in the order in which the first
// one leaves them; V is read from LDS transposed, in that same order.
#include <type_traits>

#include "fs_attn.h"

namespace fs {

namespace {

// A value that is not finite meets a probability of 0 in the rows of its tile that do not see
// it, and 0 times it is NaN.  Rows that end so, where a key that some rows do not see holds
// such values, are gone through again by whole waves, with the keys they see alone: lane j of
// 64 takes the score of key j, then each lane sums its own columns.  (4,096 rows over 32,768
// keys: 115 ms where the newest key is such a one, 2.3 where all rows see it; looking for NaN in
// the results costs nothing that shows, 2 % with 33 to 64 few rows.)
__device__ inline bool not_finite(float x) { return !(fabsf(x) < INFINITY); }

// Whether a value of the keys lo .. hi - 1 is not finite, by the whole wave.
template <bool BF, int D>
__device__ bool broken_values(const AttnArgs &a, const int32_t *table, uint32_t head, int32_t lo,
                              int32_t hi) {
  constexpr short kAll = BF ? 0x7f80 : 0x7c00;  // the exponent of what is not
  bool any = false;
  int32_t code = 0;
  for (int32_t j = lo + int32_t(threadIdx.x & 63); j < hi; j += 64) {
    const uint64_t at = 2 * row_at(a.c, __ldg(table + (j >> a.c.page_shift)), j, head, code);
#pragma unroll 4
    for (int c = 0; c < D / 8; ++c) {
      const s16x8 v = *reinterpret_cast<const s16x8 *>(a.c.v + at + c * 16);
#pragma unroll
      for (int i = 0; i < 8; ++i) any |= (v[i] & kAll) == kAll;
    }
  }
  return __any(any);
}

// Keys that one row sees of a split: `first` of them from a0 on, then those of b0 .. .
struct RowKeys {
  int32_t a0, first, b0, n;
  __device__ int32_t key(int32_t i) const { return i < first ? a0 + i : b0 + (i - first); }
};
// Those of the places lo .. hi - 1 for the row at `pos` (without sinks places are keys).
template <bool SINK>
__device__ RowKeys row_keys(const AttnArgs &a, const KeyRange &kr, int32_t lo, int32_t hi,
                            int32_t pos) {
  RowKeys r;
  if constexpr (!SINK) {
    r.a0 = r.first = 0;
    r.b0 = a.window ? max(lo, pos - a.window + 1) : lo;
    r.n = max(0, min(hi, pos + 1) - r.b0);
  } else {
    const int32_t end = lo < hi ? min(kr.key(hi - 1), pos) + 1 : 0;
    r.a0 = kr.key(lo);
    r.first = max(0, min(end, a.sinks) - r.a0);
    r.b0 = max(max(lo < kr.sink ? kr.lo : r.a0, a.sinks), pos - a.window + 1);
    r.n = r.first + max(0, end - r.b0);
  }
  return r;
}

// The keys `keys` (each seen) for one row and head, by the whole wave: the exponentials' sum
// l and reference m, and the products' sums of this lane's columns D / 64 lane .. .
template <bool BF, int D>
__device__ void row_by_key(const AttnArgs &a, const int32_t *table, uint32_t head, const short *q,
                           const RowKeys &keys, float (&acc)[D / 64], float &m, float &l) {
  constexpr int N = D / 64;
  typedef __attribute__((ext_vector_type(N))) short Cols;
  const int lane = threadIdx.x & 63;
  int32_t code = 0;
  m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) acc[i] = 0.f;
#pragma unroll 1
  for (int32_t j0 = 0; j0 < keys.n; j0 += 64) {
    const int32_t j = keys.key(min(j0 + lane, keys.n - 1));
    const uint64_t at = 2 * row_at(a.c, __ldg(table + (j >> a.c.page_shift)), j, head, code);
    float s = 0.f;
#pragma unroll 8
    for (int c = 0; c < D / 8; ++c) {
      const s16x8 kv = *reinterpret_cast<const s16x8 *>(a.c.k + at + c * 16);
      const s16x8 qv = *reinterpret_cast<const s16x8 *>(q + c * 8);
#pragma unroll
      for (int i = 0; i < 8; ++i) s = fmaf(to_f32<BF>(qv[i]), to_f32<BF>(kv[i]), s);
    }
    s = j0 + lane >= keys.n ? -INFINITY : a.flip ? -s : s;
    float top = fmaxf(m, s);
#pragma unroll
    for (int w = 32; w; w >>= 1) top = fmaxf(top, __shfl_xor(top, w, 64));
    const float f = part_factor(m, top, a.c2), mc = reference(top, a.c2) - kLift<BF>;
    const float p = exp2_fast(fmaf(s, a.c2, -mc));
    float sum = p;
#pragma unroll
    for (int w = 32; w; w >>= 1) sum += __shfl_xor(sum, w, 64);
    l = l * f + sum;
    m = top;
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] *= f;
    // (a key past the last is the last one, which the row sees, with a weight of 0)
#pragma unroll 1
    for (int k0 = 0; k0 < 64; k0 += 16) {
      if (j0 + k0 >= keys.n) break;
      Cols v[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const uint32_t lo32 = __builtin_amdgcn_readlane(int(at), k0 + k),
                       hi32 = __builtin_amdgcn_readlane(int(at >> 32), k0 + k);
        v[k] = reinterpret_cast<const Cols *>(a.c.v + (uint64_t(hi32) << 32 | lo32))[lane];
      }
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const float pk = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(p), k0 + k));
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = fmaf(pk, to_f32<BF>(v[k][i]), acc[i]);
      }
    }
  }
}

// The same, written: to out and lse, or as partial results (o, ml) at idx.
template <bool BF, int D>
__device__ void put_row_by_key(const AttnArgs &a, const int32_t *table, uint32_t head, int32_t t,
                               int32_t h, const RowKeys &keys, bool single, float *o, float *ml,
                               int64_t idx) {
  const int lane = threadIdx.x & 63;
  float acc[D / 64], top, sum;
  row_by_key<BF, D>(a, table, head, a.q + t * a.q_stride + h * D, keys, acc, top, sum);
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const int col = lane * (D / 64) + i;
    if (single)
      a.out[t * a.out_stride + h * D + col] = to_16<BF>(sum > 0.f ? acc[i] / sum : 0.f);
    else
      o[idx * D + col] = acc[i];
  }
  if (lane) return;
  if (single && a.lse) a.lse[int64_t(t) * a.n_heads + h] = log_sum(top, sum, a.c2, kLift<BF>);
  if (!single) ml[idx * 2] = top, ml[idx * 2 + 1] = sum;
}

// ---- few rows: NT tiles of 16 rows, WAVES waves.  SINK: the first keys stay visible beyond a
// window; lo, hi and what counts between them are then places of the keys seen (KeyRange), and
// a tile may hold the last sinks beside the window's first keys.  (64 requests of up to 16,384
// tokens, a window of 1,000 and 4 sinks: 25.5 us, 4.1 TB/s.)
template <bool BF, int D, int NT, int WAVES, bool SINK>
__device__ __forceinline__ void attn_few(const AttnArgs &a, int block, short *lds) {
  constexpr int KS = D / 32;  // matrix steps of a score
  constexpr int DB = D / 16;  // 16-column blocks of an output row
  constexpr int CH = D / 8;   // 16-byte chunks of a key row
  constexpr int RW = 64 / CH, LD = 32 / RW;  // rows of a wave's load, loads of 32 keys' K (or V)
  constexpr int kIds = 512;   // page ids kept in LDS
  constexpr bool kTwoParts = NT <= 2;  // of a probability
  auto kv_lds = reinterpret_cast<short(*)[2][32 * D]>(lds);  // a wave's K and V
  __shared__ float wm[WAVES][NT * 16], wl[WAVES][NT * 16];
  __shared__ uint32_t ids[kIds];
  __shared__ uint32_t broken[NT * 16];  // a row to be gone through again
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, g4 = lane >> 4;
  // Work-groups go to the 8 dies in turn: heads fastest, and each split shifts the
  // requests by one, so a long request's splits do not gather on one die.
  const int hk = block % a.c.n_kv_heads, sz = block / a.c.n_kv_heads;
  const int z = sz / a.n_seqs, s = (sz + z) % a.n_seqs;
  const int32_t q0 = __ldg(a.q_off + s), n = __ldg(a.q_off + s + 1) - q0;
  const int G = a.group, R = n * G;
  if (R <= 0 || R > kFewRows) return;
  int32_t code = 0;
  const int32_t kv = checked_len(a.kv_len, s, a.max_kv, code);
  const KeyRange kr = key_range(a, n, kv, 0, n - 1);
  const int32_t from0 = SINK ? 0 : kr.lo, to0 = SINK ? kr.length() : kr.hi;
  const bool single = to0 - from0 <= a.few_split;
  const int32_t lo = from0 + z * a.few_split;
  if (z > 0 && lo >= to0) return;
  const int32_t hi = min(to0, lo + a.few_split);
  auto key = [&](int32_t place) { return SINK ? kr.key(place) : place; };
  const int32_t *table = a.c.table + s * a.c.table_stride;
  const uint32_t head = hk * a.c.head_stride;

  // queries: row r16 of each tile, this lane's 8 elements of each step
  s16x8 qf[NT][KS];
  int32_t pos[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int r = min(t * 16 + r16, R - 1), tok = r / G, h = hk * G + (r - tok * G);
    pos[t] = t * 16 + r16 < R ? kv - n + tok : -1;
    const short *qp = a.q + (q0 + tok) * a.q_stride + h * D + g4 * 8;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      qf[t][k] = *reinterpret_cast<const s16x8 *>(qp + k * 32);
      if (a.flip) qf[t][k] ^= short(0x8000);
    }
  }
  f32x4 o[NT][DB] = {};
  float m[NT], l[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) m[t] = -INFINITY, l[t] = 0.f;

  // This lane's row and 16-byte chunk of each load.  (Straight into registers in the matrix
  // cores' layout, 16 lanes would touch 16 rows: a quarter of the cache's rate.)
  uint32_t lcol[LD];
#pragma unroll
  for (int i = 0; i < LD; ++i) {
    const int r = i * RW + lane / CH;
    lcol[i] = head + (tile_at<D>(r, lane % CH) - r * D);
  }
  const uint32_t to = lds_address(kv_lds[wave][0]);

  // the ids of up to kIds pages at a time
  for (int32_t from = lo; from < hi;) {
    const PageIds span = page_ids<SINK>(kr, from, hi, a.c.page_shift, kIds);
    const int32_t end = span.end;
    __syncthreads();
    for (int i = tid; i < span.n; i += WAVES * 64) {
      const uint32_t page = __ldg(table + span.page(i));
      if (page >= a.c.n_pages) code = FS_E_RANGE;
      ids[i] = page < a.c.n_pages ? page : 0;
    }
    __syncthreads();
    // the waves take 32 keys in turn
    const int32_t first = from + wave * 32;
    const int32_t tiles = first < end ? (end - first + WAVES * 32 - 1) / (WAVES * 32) : 0;
    auto issue = [&](int32_t t) {
      const int32_t j0 = first + t * (WAVES * 32);
      uint64_t at[LD];
#pragma unroll
      for (int i = 0; i < LD; ++i) {
        const int32_t j = key(min(j0 + i * RW + lane / CH, end - 1));
        at[i] = 2 * row_at(a.c, ids[span.slot(j)], j, lcol[i], code);
      }
#pragma unroll
      for (int i = 0; i < LD; ++i) load_to_lds(a.c.k + at[i], to + i * 1024);
#pragma unroll
      for (int i = 0; i < LD; ++i) load_to_lds(a.c.v + at[i], to + 32 * D * 2 + i * 1024);
    };
    if (tiles > 0) issue(0);
    for (int32_t t = 0; t < tiles; ++t) {
      const int32_t j0 = first + t * (WAVES * 32);
      wait_own<0>();
      const short *kb = kv_lds[wave][0], *vb = kv_lds[wave][1];
      f32x4 sc[NT][2] = {};
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const s16x8 kf =
              *reinterpret_cast<const s16x8 *>(kb + tile_at<D>(b * 16 + r16, k * 4 + g4));
#pragma unroll
          for (int r = 0; r < NT; ++r) sc[r][b] = mfma_16x16x32<BF>(kf, qf[r][k], sc[r][b]);
        }
      s16x8 pf[NT], pl[NT];
#pragma unroll
      for (int r = 0; r < NT; ++r) {
        float p[8], top = -INFINITY;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int32_t v = j0 + b * 16 + g4 * 4 + i, j = key(v);
            const bool see = j <= pos[r] && v < end &&
                             (a.window == 0 || j > pos[r] - a.window || (SINK && j < a.sinks));
            p[b * 4 + i] = see ? sc[r][b][i] : -INFINITY;
            top = fmaxf(top, p[b * 4 + i]);
          }
        top = max_of_halves(fmaxf(top, __shfl_xor(top, 16, 64)));
        const float m2 = fmaxf(m[r], top);
        // (-inf less -inf is no number and asks for nothing)
        if (__any((m2 - m[r]) * a.c2 > kSlack)) {
          const float f = m[r] == -INFINITY ? 0.f : part_factor(m[r], m2, a.c2);
          l[r] *= f;
#pragma unroll
          for (int d = 0; d < DB; ++d) o[r][d] *= f;
          m[r] = m2;
        }
        const float mc = reference(m[r], a.c2) - kLift<BF>;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[i] = exp2_fast(fmaf(p[i], a.c2, -mc));
          l[r] += p[i];
        }
        pf[r] = pack8<BF>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (kTwoParts) pl[r][i] = to_16<BF>(p[i] - to_f32<BF>(pf[r][i]));
      }
      // keys 4 g4 .. + 3 and 16 + 4 g4 .. + 3 of the tile, 16 columns at a time
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        const int row = 4 * g4 + (r16 >> 2), col = d * 16 + (r16 & 3) * 4;
        const s16x4 v0 = read_tr(vb + tile_at<D>(row, col >> 3) + (col & 7));
        const s16x4 v1 = read_tr(vb + tile_at<D>(row + 16, col >> 3) + (col & 7));
        const s16x8 vv = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int r = 0; r < NT; ++r) {
          o[r][d] = mfma_16x16x32<BF>(vv, pf[r], o[r][d]);
          if (kTwoParts) o[r][d] = mfma_16x16x32<BF>(vv, pl[r], o[r][d]);
        }
      }
      if (t + 1 < tiles) {
        reads_done();
        issue(t + 1);
      }
    }
    from = end;
  }
  raise_err(a.err, code);

  // the waves' results, joined in LDS a tile of rows at a time
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    l[t] += __shfl_xor(l[t], 16, 64);
    l[t] += __shfl_xor(l[t], 32, 64);
    if (g4 == 0) wm[wave][t * 16 + r16] = m[t], wl[wave][t * 16 + r16] = l[t];
  }
  bool any = false;
  if (n > 1 && tid < NT * 16) broken[tid] = 0;
  float *buf = reinterpret_cast<float *>(kv_lds);  // [WAVES][16][D / 2]: half of the columns
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (t * 16 >= R) break;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      __syncthreads();
#pragma unroll
      for (int d = 0; d < DB / 2; ++d)
        *reinterpret_cast<f32x4 *>(
            buf + (wave * 16 + r16) * (D / 2) + ((d * 16 + g4 * 4) ^ ((r16 & 3) * 4))) =
            o[t][half * (DB / 2) + d];
      __syncthreads();
      for (int e = tid; e < 16 * D / 8; e += WAVES * 64) {
        const int r = e / (D / 8), col = (e - r * (D / 8)) * 4;
        if (t * 16 + r >= R) continue;
        const int tr = t * 16 + r;
        float top = wm[0][tr];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) top = fmaxf(top, wm[w][tr]);
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
          const float f = part_factor(wm[w][tr], top, a.c2);
          sum += f * wl[w][tr];
          acc += f * *reinterpret_cast<const f32x4 *>(buf + (w * 16 + r) * (D / 2) +
                                                      (col ^ ((r & 3) * 4)));
        }
        const int tok = tr / G, h = hk * G + (tr - tok * G), cc = half * (D / 2) + col;
        if (single) {
          const float inv = sum > 0.f ? 1.f / sum : 0.f;
          s16x4 v;
          acc *= inv;
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = to_16<BF>(acc[i]);
          *reinterpret_cast<s16x4 *>(a.out + (q0 + tok) * a.out_stride + h * D + cc) = v;
          if (cc == 0 && a.lse)
            a.lse[int64_t(q0 + tok) * a.n_heads + h] = log_sum(top, sum, a.c2, kLift<BF>);
        } else {
          const int64_t idx =
              ((int64_t(z) * a.n_seqs + s) * a.few_tokens + tok) * a.n_heads + h;
          *reinterpret_cast<f32x4 *>(a.few_o + idx * D + cc) = acc;
          if (cc == 0) a.few_ml[idx * 2] = top, a.few_ml[idx * 2 + 1] = sum;
        }
        if (n > 1 && !not_finite(sum)) {
          float zero = 0.f;  // NaN where a result is not finite
#pragma unroll
          for (int i = 0; i < 4; ++i) zero = fmaf(acc[i], 0.f, zero);
          if (zero != 0.f) broken[tr] = 1, any = true;
        }
      }
    }
  }
  if (n == 1 || !__syncthreads_or(any)) return;  // (one token's rows see every key)
  if constexpr (SINK) {  // (all keys of the split: a superset of the hidden ones)
    if (!broken_values<BF, D>(a, table, head, lo, min(hi, kr.sink)) &&
        !broken_values<BF, D>(a, table, head, key(max(lo, kr.sink)), key(hi - 1) + 1))
      return;
  } else if (!broken_values<BF, D>(a, table, head, max(lo, kv - n + 1), hi) &&
             !(a.window && broken_values<BF, D>(a, table, head, lo, min(hi, kv - a.window)))) {
    return;
  }
  wait_own<0>();  // what was stored above comes first
  __syncthreads();
#pragma unroll 1
  for (int r = wave; r < R; r += WAVES) {
    if (!broken[r]) continue;
    const int tok = r / G, h = hk * G + (r - tok * G);
    put_row_by_key<BF, D>(a, table, head, q0 + tok, h,
                          row_keys<SINK>(a, kr, lo, hi, kv - n + tok), single, a.few_o, a.few_ml,
                          ((int64_t(z) * a.n_seqs + s) * a.few_tokens + tok) * a.n_heads + h);
  }
}

// ---- chunks: WAVES waves of 32 rows, 64 keys at a time through two buffers
template <bool BF, int D, int WAVES, bool SINK>
__device__ __forceinline__ void attn_chunk(const AttnArgs &a, int block, int z, short *lds) {
  constexpr int KS = D / 16;       // matrix steps of a score
  constexpr int DB = D / 32;       // 32-column blocks of an output row
  constexpr int CH = D / 8;        // 16-byte chunks of a key row
  constexpr int RW = 64 / CH;      // rows of a wave's load
  constexpr int LD = 64 / WAVES / RW;  // a wave's loads of K, and of V, for 64 keys
  static_assert(LD >= 1, "a wave loads whole rows");
  auto kt = reinterpret_cast<short(*)[64 * D]>(lds), vt = kt + 2;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r32 = lane & 31, h2 = lane >> 5;
  const int hk = block % a.c.n_kv_heads;
  int32_t s, r0;
  chunk_tile(a, block / a.c.n_kv_heads, s, r0);
  const int32_t q0 = __ldg(a.q_off + s), n = __ldg(a.q_off + s + 1) - q0;
  const int G = a.group, R = n * G;
  if (r0 < 0 || R <= kFewRows) return;
  int32_t code = 0;
  const int32_t kv = checked_len(a.kv_len, s, a.max_kv, code);
  const KeyRange kr = key_range(a, n, kv, r0 / G, (min(r0 + WAVES * 32, R) - 1) / G);
  const int32_t from0 = SINK ? 0 : kr.lo, to0 = SINK ? kr.length() : kr.hi;
  const bool single = to0 - from0 <= a.chunk_split;
  const int32_t lo = from0 + z * a.chunk_split;
  if (z > 0 && lo >= to0) return;
  const int32_t hi = min(to0, lo + a.chunk_split);
  auto key = [&](int32_t place) { return SINK ? kr.key(place) : place; };
  const int32_t *table = a.c.table + s * a.c.table_stride;
  const uint32_t head = hk * a.c.head_stride;

  const int row = r0 + wave * 32 + r32;
  const int tok = min(row, R - 1) / G, h = hk * G + (min(row, R - 1) - tok * G);
  const int32_t pos = kv - n + tok;
  // the wave's first and last row, and the first key that its last row's window leaves
  const int32_t pos_lo = kv - n + min(r0 + wave * 32, R - 1) / G;
  const int32_t win_hi =
      a.window ? kv - n + min(r0 + wave * 32 + 31, R - 1) / G - a.window : INT32_MIN;
  s16x8 qf[KS];
  {
    const short *qp = a.q + (q0 + tok) * a.q_stride + h * D + h2 * 8;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      qf[k] = *reinterpret_cast<const s16x8 *>(qp + k * 16);
      if (a.flip) qf[k] ^= short(0x8000);
    }
  }
  f32x16 o[DB] = {};
  float m = -INFINITY, l = 0.f;
  bool hidden = false;  // from some row of the wave, some key

  // This lane's row and 16-byte chunk of each of the wave's loads, RW rows at a time.
  int32_t lrow[LD];
  uint32_t lcol[LD], page[LD];
#pragma unroll
  for (int i = 0; i < LD; ++i) {
    lrow[i] = (wave * LD + i) * RW + lane / CH;
    lcol[i] = head + (tile_at<D>(lrow[i], lane % CH) - lrow[i] * D);
  }
  // page ids are loaded one tile ahead of the rows
  auto pages = [&](int32_t j0) {
#pragma unroll
    for (int i = 0; i < LD; ++i)
      page[i] = __ldg(table + (key(min(j0 + lrow[i], hi - 1)) >> a.c.page_shift));
  };
  const uint32_t k_to = lds_address(kt[0] + wave * LD * RW * D),
                 v_to = lds_address(vt[0] + wave * LD * RW * D);
  auto issue = [&](int32_t j0, int buf) {
    // all ids are waited for here: a wait between the loads would be for those loads too
#pragma unroll
    for (int i = 0; i < LD; ++i) asm volatile("" : "+v"(page[i]));
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const uint64_t at =
          2 * row_at(a.c, page[i], key(min(j0 + lrow[i], hi - 1)), lcol[i], code);
      load_to_lds(a.c.k + at, k_to + (buf * 64 + i * RW) * D * 2);
      load_to_lds(a.c.v + at, v_to + (buf * 64 + i * RW) * D * 2);
    }
  };
  if (lo < hi) {
    pages(lo);
    issue(lo, 0);
    pages(lo + 64);
  }
  int buf = 0;
  for (int32_t j0 = lo; j0 < hi; j0 += 64, buf ^= 1) {
    wait_loads<0>();
    if (j0 + 64 < hi) {
      issue(j0 + 64, buf ^ 1);
      pages(j0 + 128);
    }
    const short *kb = kt[buf], *vb = vt[buf];
    f32x16 sc[2] = {};
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int c = 0; c < 2; ++c)
        sc[c] = mfma_32x32x16<BF>(
            *reinterpret_cast<const s16x8 *>(kb + tile_at<D>(c * 32 + r32, k * 2 + h2)), qf[k],
            sc[c]);
    // keys that some row of the wave does not see
    if (key(j0 + 63) > pos_lo || j0 + 64 > hi || key(j0) <= win_hi) {
      hidden = true;
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int32_t v = j0 + c * 32 + 8 * (i >> 2) + 4 * h2 + (i & 3), j = key(v);
          if (j > pos || v >= hi ||
              (a.window && j <= pos - a.window && !(SINK && j < a.sinks)))
            sc[c][i] = -INFINITY;
        }
    }
    float top = sc[0][0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, sc[0][i]);
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[1][i]);
    const float m2 = fmaxf(m, max_of_halves(top));
    if (__any((m2 - m) * a.c2 > kSlack)) {
      const float f = m == -INFINITY ? 0.f : part_factor(m, m2, a.c2);
      l *= f;
#pragma unroll
      for (int d = 0; d < DB; ++d) o[d] *= f;
      m = m2;
    }
    const float mc = reference(m, a.c2) - kLift<BF>;
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[i] = exp2_fast(fmaf(sc[c][u * 8 + i], a.c2, -mc));
          l += p[i];
        }
        const s16x8 pf = pack8<BF>(p);
        // keys 4 h2 .. + 3 and 8 + 4 h2 .. + 3 of this 16
        const int vr = c * 32 + u * 16 + 4 * h2 + ((lane & 15) >> 2);
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const int col = d * 32 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
          const s16x4 v0 = read_tr(vb + tile_at<D>(vr, col >> 3) + (col & 7));
          const s16x4 v1 = read_tr(vb + tile_at<D>(vr + 8, col >> 3) + (col & 7));
          o[d] = mfma_32x32x16<BF>(__builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7), pf,
                                   o[d]);
        }
      }
  }
  raise_err(a.err, code);
  l += __shfl_xor(l, 32, 64);
  float zero = 0.f;  // NaN once a result is not finite
  if (row < R) {
    if (single) {
      const float inv = l > 0.f ? 1.f / l : 0.f;
      short *op = a.out + (q0 + tok) * a.out_stride + h * D;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s16x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = o[d][i * 4 + e] * inv;
            zero = fmaf(x, 0.f, zero);
            v[e] = to_16<BF>(x);
          }
          *reinterpret_cast<s16x4 *>(op + d * 32 + i * 8 + h2 * 4) = v;
        }
      if (h2 == 0 && a.lse)
        a.lse[int64_t(q0 + tok) * a.n_heads + h] = log_sum(m, l, a.c2, kLift<BF>);
    } else {
      const int64_t idx = (int64_t(z) * a.rows + q0 + tok) * a.n_heads + h;
      float *op = a.chunk_o + idx * D;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 x = {o[d][i * 4], o[d][i * 4 + 1], o[d][i * 4 + 2], o[d][i * 4 + 3]};
#pragma unroll
          for (int e = 0; e < 4; ++e) zero = fmaf(x[e], 0.f, zero);
          *reinterpret_cast<f32x4 *>(op + d * 32 + i * 8 + h2 * 4) = x;
        }
      if (h2 == 0) a.chunk_ml[idx * 2] = m, a.chunk_ml[idx * 2 + 1] = l;
    }
  }
  if (!hidden) return;
  uint64_t again = __ballot(zero != 0.f && !not_finite(l));
  again = (again | again >> 32) & 0xffffffffu;  // rows of the wave
  if (!again) return;
  if constexpr (SINK) {  // (all keys of the split: a superset of the hidden ones)
    if (!broken_values<BF, D>(a, table, head, lo, min(hi, kr.sink)) &&
        !broken_values<BF, D>(a, table, head, key(max(lo, kr.sink)), key(hi - 1) + 1))
      return;
  } else if (!broken_values<BF, D>(a, table, head, max(lo, pos_lo + 1), hi) &&
             !(a.window && broken_values<BF, D>(a, table, head, lo, min(hi, win_hi + 1)))) {
    return;
  }
  wait_own<0>();  // what was stored above comes first
#pragma unroll 1
  for (; again; again &= again - 1) {
    const int r = r0 + wave * 32 + __builtin_ctzll(again), t = r / G, hh = hk * G + (r - t * G);
    put_row_by_key<BF, D>(a, table, head, q0 + t, hh, row_keys<SINK>(a, kr, lo, hi, kv - n + t),
                          single, a.chunk_o, a.chunk_ml, (int64_t(z) * a.rows + q0 + t) * a.n_heads + hh);
  }
}

template <bool BF, int D, int NT, int WAVES, bool SINK>
__global__ void __launch_bounds__(WAVES * 64) k_attn_few(AttnArgs a) {
  __shared__ __align__(16) short lds[WAVES * 64 * D];
  attn_few<BF, D, NT, WAVES, SINK>(a, blockIdx.x, lds);
}
template <bool BF, int D, int WAVES, bool SINK>
__global__ void __launch_bounds__(WAVES * 64, 2) k_attn_chunk(AttnArgs a) {
  __shared__ __align__(16) short lds[256 * D];
  attn_chunk<BF, D, WAVES, SINK>(a, blockIdx.x, blockIdx.y, lds);
}
// Both kinds of requests in one launch: the single tokens' loads fill what the chunks' last
// work-groups leave of the card.  (24 requests of up to 8,192 tokens, 16 heads of 64, a window
// of 3,000: 82 us, 99 one after the other, 102 with the chunks last; 24 of up to 16,000, most
// of them chunks of 400 or less: 216 us, 232 one after the other, 301 with the chunks last,
// 275 with the two evenly mixed.)
template <bool BF, int D, int NT, bool SINK>
__global__ void __launch_bounds__(256, 2) k_attn_mixed(AttnArgs a, int chunk, int tiles) {
  __shared__ __align__(16) short lds[256 * D];
  const int block = blockIdx.x;
  if (block < chunk)
    attn_chunk<BF, D, 4, SINK>(a, block % tiles, block / tiles, lds);
  else
    attn_few<BF, D, NT, 4, SINK>(a, block - chunk, lds);
}

template <bool BF, int D, bool SINK>
void run(const AttnArgs &a, const Plan &p, hipStream_t stream) {
  const dim3 block(256);
  const int few = p.few_seqs > 0 ? a.n_seqs * a.c.n_kv_heads * p.few_splits : 0;
  const int tiles = p.chunk_tiles * a.c.n_kv_heads;
  const int chunk = p.chunk_seqs > 0 ? tiles * p.chunk_splits : 0;
  // In one launch where one kernel holds both without spilling registers.
  const bool mixed = few > 0 && chunk > 0 && p.chunk_rows == 128 && (D == 64 || p.few_rows <= 32);
  auto by_rows = [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    if constexpr (D == 64 || NT <= 2)
      if (mixed)
        hipLaunchKernelGGL((k_attn_mixed<BF, D, NT, SINK>), dim3(chunk + few), block, 0, stream, a, chunk,
                           tiles);
    if constexpr (NT <= 2)
      if (p.few_waves == 8)
        hipLaunchKernelGGL((k_attn_few<BF, D, NT, 8, SINK>), dim3(few), dim3(512), 0, stream, a);
    if (few > 0 && !mixed && p.few_waves == 4)
      hipLaunchKernelGGL((k_attn_few<BF, D, NT, 4, SINK>), dim3(few), block, 0, stream, a);
  };
  if (p.few_rows <= 16)
    by_rows(std::integral_constant<int, 1>());
  else if (p.few_rows <= 32)
    by_rows(std::integral_constant<int, 2>());
  else
    by_rows(std::integral_constant<int, 4>());
  if (chunk > 0 && !mixed) {
    const dim3 grid(tiles, p.chunk_splits);
    if constexpr (D == 128)
      if (p.chunk_rows == 256)
        hipLaunchKernelGGL((k_attn_chunk<BF, D, 8, SINK>), grid, dim3(512), 0, stream, a);
    if (p.chunk_rows == 128)
      hipLaunchKernelGGL((k_attn_chunk<BF, D, 4, SINK>), grid, block, 0, stream, a);
  }
  if (p.few_splits > 1)
    hipLaunchKernelGGL((k_attn_join_few<BF, D>), dim3(a.n_heads, a.n_seqs, p.few_tokens), block, 0,
                       stream, a);
  if (p.chunk_splits > 1) {
    const int64_t lanes = int64_t(a.rows) * a.n_heads * (D / 4);
    hipLaunchKernelGGL((k_attn_join_chunk<BF, D>), dim3((lanes + 255) / 256), block, 0, stream, a);
  }
}

constexpr int32_t kOnceSinks = 1024;

// Without a window, or with one that no length can fill, sinks are none: the call is then
// fs_paged_attention's, split as ever, and its sums are taken in the same order.
Shape shape16(const fs_step *s, const fs_kv_cache *c, int32_t n_heads, int32_t window,
              int32_t sinks) {
  Shape sh = shape_of(s, n_heads, c->n_kv_heads, c->head_dim, window, sinks, 1024, 131072, 0, 512, 1024);
  if (sh.sinks > 0) sh.few_once = kOnceSinks;
  return sh;
}

}  // namespace

size_t attention_workspace_bytes(const fs_step *s, const fs_kv_cache *c, int32_t n_heads,
                                 int32_t window, int32_t sinks) {
  const Shape sh = shape16(s, c, n_heads, window, sinks);
  return space(plan(s, sh), s, sh).total();
}

hipError_t launch_attention(const fs_step *s, const fs_kv_cache *c, int32_t n_heads, float scale,
                            int32_t window, int32_t sinks, const void *q, int64_t q_stride,
                            void *out, int64_t out_stride, float *lse, void *ws, int32_t *err,
                            hipStream_t stream) {
  const Shape sh = shape16(s, c, n_heads, window, sinks);
  const Plan p = plan(s, sh);
  AttnArgs a;
  fill_args(a, p, space(p, s, sh), sh, s, scale, q, q_stride, out, out_stride, lse, ws, err);
  a.c = dev_cache(c);
  a.lift = c->dtype == FS_BF16 ? kLift<true> : kLift<false>;
  auto go = [&](auto bf, auto dim) {
    constexpr bool BF = decltype(bf)::value;
    constexpr int D = decltype(dim)::value;
    if (sh.sinks > 0)
      run<BF, D, true>(a, p, stream);
    else
      run<BF, D, false>(a, p, stream);
  };
  const std::integral_constant<int, 64> d64;
  const std::integral_constant<int, 128> d128;
  if (c->dtype == FS_BF16)
    c->head_dim == 128 ? go(std::true_type(), d128) : go(std::true_type(), d64);
  else
    c->head_dim == 128 ? go(std::false_type(), d128) : go(std::false_type(), d64);
  return hipGetLastError();
}

}  // namespace fs
