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
//                 PFLOP/s, 1.84 to 2.04 ms from card to card; head_dim 64: 0.84 PFLOP/s).  128 or 256 rows a work-group share each tile
//                 of 64 keys.
//   k_attn_join_* join the splits' results with their maxima and sums, in split order.
// Both products run with the keys as rows of the first operand (S^T = K Q^T,
// O^T = V^T P^T): a lane then holds scores of one query row only, its probabilities are
// the second product's operand as they lie in registers, and the running factors are one
// number per lane.  The second product takes the keys in the order in which the first
// one leaves them; V is read from LDS transposed, in that same order.
#include <type_traits>

#include "fs_engine.h"

namespace fs {

namespace {

constexpr int kFewRows = 64;    // rows (tokens times group) that k_attn_few takes
constexpr int64_t kMostPartial = int64_t(1) << 28;  // bytes of partial results, about
constexpr float kLn2 = 0.693147180559945309f;

struct AttnArgs {
  const int32_t *q_off, *kv_len;
  int32_t n_seqs, max_kv, rows, n_heads, window, group;
  DevCache c;
  const short *q;
  short *out;
  int64_t q_stride, out_stride;
  float *lse;
  float c2;            // |scale| * log2(e)
  uint32_t flip;       // sign of the scale, applied to the queries
  int32_t few_split;   // keys of a split (k_attn_few)
  int32_t few_tokens;  // most tokens of a request that k_attn_few takes
  int32_t chunk_rows;  // rows of a work-group of k_attn_chunk
  int32_t chunk_split;
  float *few_o, *few_ml;      // [splits][n_seqs][few_tokens][heads][D], [..][2]
  float *chunk_o, *chunk_ml;  // [splits][rows][heads][D], [..][2]
  int32_t *err;
};

// Keys that the tokens tok0 .. tok1 of a request with n new and kv cached ones see.
struct KeyRange {
  int32_t lo, hi;
};
__device__ inline KeyRange key_range(const AttnArgs &a, int32_t n, int32_t kv, int32_t tok0,
                                     int32_t tok1) {
  KeyRange r;
  r.lo = a.window ? max(0, kv - n + tok0 - a.window + 1) : 0;
  r.hi = max(0, kv - n + tok1 + 1);
  return r;
}

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
// Four keys by sixteen columns of V per 16 lanes, transposed: lane i of the 16 names the
// 8 bytes (key i / 4, columns 4 (i % 4) ..) and gets column i of the four keys.
__device__ inline s16x4 read_tr(const short *p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (lds_s16x4 *)(__attribute__((address_space(3))) short *)(p));
}

// Where 16-byte chunk `c` of key row `r` lies in an LDS tile with D-element rows: chunks
// are exchanged so that 16 rows' chunks, and 4 rows' transposed reads, fall on different
// banks.
template <int D>
__device__ inline int tile_at(int r, int c) {
  if constexpr (D == 128)
    return r * 128 + ((c ^ ((r & 3) << 2 | ((r >> 2) & 3))) * 8);
  else
    return r * 64 + ((c ^ (((r >> 1) & 1) << 2 | ((r >> 2) & 3))) * 8);
}

// Probabilities enter the second product in 16 bits.  Up to 32 few rows, where the bytes of the
// cache are the bound, as the sum of two values: the error against 64 bits is that of rounding
// the result alone (64 requests of up to 16,384 tokens 122.4 us, 122.0 with one value; 32
// requests of 32 rows 119 and 118).  In k_attn_chunk and for more few rows as one value, with
// 1.1 to 1.4 times that error: a second product would take 4,096 rows over 32,768 keys from
// 1.92 to 2.65 ms, 24 mixed requests from 89 to 113 us, 32 of 64 rows from 180 to 192.
template <bool BF>
__device__ inline s16x8 pack8(const float *p) {
  s16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = to_16<BF>(p[i]);
  return v;
}

// A row keeps the reference of its exponentials until a score passes it by 2^kSlack, so
// that its sums are seldom scaled; probabilities then reach 2^kSlack, which costs no
// precision.
constexpr float kSlack = 8.f;
// In half precision the exponentials count in units of 2^-kLift (sums and products alike, so
// that it cancels): with kSlack they stay below 2^16, and a probability is lost to the type's
// smallest number from 2^-32 of the reference on, not from 2^-25.  (No change in time.)
template <bool BF>
constexpr float kLift = BF ? 0.f : 7.f;

// The larger of the two halves' values, in both.
__device__ inline float max_of_halves(float x) {
  const uint32_t b = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// A reference of the exponentials as they use it: 0 while there is none and where it is
// infinite, so that a score of inf makes the sum inf (inf - inf would make it NaN).
__device__ inline float reference(float m, float c2) {
  return fabsf(m) == INFINITY ? 0.f : m * c2;
}
// What a part with the maximum m weighs where the largest of the parts' is `top` (inf less
// inf is no number; a part without a maximum holds sums of 0).
__device__ inline float part_factor(float m, float top, float c2) {
  return exp2_fast(m == top ? 0.f : (m - top) * c2);
}
// ln of a row's sum of exponentials: -inf only where nothing was summed (a NaN score makes
// the sum NaN, one of inf makes it inf).
template <bool BF>
__device__ inline float log_sum(float top, float sum, float c2) {
  return sum == 0.f ? -INFINITY : (top * c2 + (__log2f(sum) - kLift<BF>)) * kLn2;
}

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

// Keys lo .. hi - 1 (each seen) for one row and head, by the whole wave: the exponentials' sum
// l and reference m, and the products' sums of this lane's columns D / 64 lane .. .
template <bool BF, int D>
__device__ void row_by_key(const AttnArgs &a, const int32_t *table, uint32_t head, const short *q,
                           int32_t lo, int32_t hi, float (&acc)[D / 64], float &m, float &l) {
  constexpr int N = D / 64;
  typedef __attribute__((ext_vector_type(N))) short Cols;
  const int lane = threadIdx.x & 63;
  int32_t code = 0;
  m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) acc[i] = 0.f;
#pragma unroll 1
  for (int32_t j0 = lo; j0 < hi; j0 += 64) {
    const int32_t j = min(j0 + lane, hi - 1);
    const uint64_t at = 2 * row_at(a.c, __ldg(table + (j >> a.c.page_shift)), j, head, code);
    float s = 0.f;
#pragma unroll 8
    for (int c = 0; c < D / 8; ++c) {
      const s16x8 kv = *reinterpret_cast<const s16x8 *>(a.c.k + at + c * 16);
      const s16x8 qv = *reinterpret_cast<const s16x8 *>(q + c * 8);
#pragma unroll
      for (int i = 0; i < 8; ++i) s = fmaf(to_f32<BF>(qv[i]), to_f32<BF>(kv[i]), s);
    }
    s = j0 + lane >= hi ? -INFINITY : a.flip ? -s : s;
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
      if (j0 + k0 >= hi) break;
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
                               int32_t h, int32_t pos, int32_t lo, int32_t hi, bool single, float *o,
                               float *ml, int64_t idx) {
  const int lane = threadIdx.x & 63;
  float acc[D / 64], top, sum;
  row_by_key<BF, D>(a, table, head, a.q + t * a.q_stride + h * D,
                    a.window ? max(lo, pos - a.window + 1) : lo, min(hi, pos + 1), acc, top, sum);
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const int col = lane * (D / 64) + i;
    if (single)
      a.out[t * a.out_stride + h * D + col] = to_16<BF>(sum > 0.f ? acc[i] / sum : 0.f);
    else
      o[idx * D + col] = acc[i];
  }
  if (lane) return;
  if (single && a.lse) a.lse[int64_t(t) * a.n_heads + h] = log_sum<BF>(top, sum, a.c2);
  if (!single) ml[idx * 2] = top, ml[idx * 2 + 1] = sum;
}

// ---- few rows: NT tiles of 16 rows, WAVES waves
template <bool BF, int D, int NT, int WAVES>
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
  const bool single = kr.hi - kr.lo <= a.few_split;
  const int32_t lo = kr.lo + z * a.few_split;
  if (z > 0 && lo >= kr.hi) return;
  const int32_t hi = min(kr.hi, lo + a.few_split);
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

  // the page ids of up to kIds pages at a time
  for (int32_t from = lo; from < hi;) {
    const int32_t p0 = from >> a.c.page_shift;
    const int32_t end = int32_t(min(int64_t(hi), int64_t(p0 + kIds) << a.c.page_shift));
    __syncthreads();
    for (int i = tid; i < ((end - 1) >> a.c.page_shift) - p0 + 1; i += WAVES * 64) {
      const uint32_t page = __ldg(table + p0 + i);
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
        const int32_t j = min(j0 + i * RW + lane / CH, end - 1);
        at[i] = 2 * row_at(a.c, ids[(j >> a.c.page_shift) - p0], j, lcol[i], code);
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
            const int32_t j = j0 + b * 16 + g4 * 4 + i;
            const bool see = j <= pos[r] && j < end && (a.window == 0 || j > pos[r] - a.window);
            p[b * 4 + i] = see ? sc[r][b][i] : -INFINITY;
            top = fmaxf(top, p[b * 4 + i]);
          }
        top = max_of_halves(fmaxf(top, __shfl_xor(top, 16, 64)));
        const float m2 = fmaxf(m[r], top);
        // (-inf less -inf is no number and asks for nothing)
        if (__any((m2 - m[r]) * a.c2 > kSlack)) {
          const float f = m[r] == -INFINITY ? 0.f : exp2_fast((m[r] - m2) * a.c2);
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
            a.lse[int64_t(q0 + tok) * a.n_heads + h] = log_sum<BF>(top, sum, a.c2);
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
  if (!broken_values<BF, D>(a, table, head, max(lo, kv - n + 1), hi) &&
      !(a.window && broken_values<BF, D>(a, table, head, lo, min(hi, kv - a.window))))
    return;
  wait_own<0>();  // what was stored above comes first
  __syncthreads();
#pragma unroll 1
  for (int r = wave; r < R; r += WAVES) {
    if (!broken[r]) continue;
    const int tok = r / G, h = hk * G + (r - tok * G);
    put_row_by_key<BF, D>(a, table, head, q0 + tok, h, kv - n + tok, lo, hi, single, a.few_o,
                          a.few_ml,
                          ((int64_t(z) * a.n_seqs + s) * a.few_tokens + tok) * a.n_heads + h);
  }
}

// Row tile number b of k_attn_chunk, a request's last rows (which see the most keys) first.
// Up to 64 requests are taken in the order of the keys they see, the most first, so that
// the work ends evenly; more in their own order, request s owning the tile numbers from
// q_off[s] * G / chunk_rows + s on.  r0 < 0: no rows.
__device__ inline void chunk_tile(const AttnArgs &a, int32_t b, int32_t &s, int32_t &r0) {
  if (a.n_seqs <= 64) {
    const int32_t i = min(int32_t(__lane_id()), a.n_seqs - 1);
    const int32_t n = __ldg(a.q_off + i + 1) - __ldg(a.q_off + i), R = n * a.group;
    const int32_t kv = __ldg(a.kv_len + i);
    const int32_t keys = a.window ? min(kv, a.window + n) : kv;
    const int32_t mine = R > kFewRows ? (R + a.chunk_rows - 1) / a.chunk_rows : 0;
    int32_t before = 0;
    for (int j = 0; j < a.n_seqs; ++j) {
      const int32_t other = __builtin_amdgcn_readlane(keys, j);
      if (other > keys || (other == keys && j < i)) before += __builtin_amdgcn_readlane(mine, j);
    }
    const uint64_t hit =
        __ballot(int32_t(__lane_id()) < a.n_seqs && before <= b && b < before + mine);
    if (!hit) {
      s = 0;
      r0 = -1;
      return;
    }
    s = __builtin_ctzll(hit);
    r0 = (__builtin_amdgcn_readlane(mine, s) - 1 - (b - __builtin_amdgcn_readlane(before, s))) *
         a.chunk_rows;
    return;
  }
  s = last_at_most(a.n_seqs, b, [&](int32_t i) {
    return __ldg(a.q_off + i) * a.group / a.chunk_rows + i;
  });
  const int32_t q0 = __ldg(a.q_off + s), R = (__ldg(a.q_off + s + 1) - q0) * a.group;
  const int32_t tiles = (R + a.chunk_rows - 1) / a.chunk_rows;
  r0 = (tiles - 1 - (b - q0 * a.group / a.chunk_rows - s)) * a.chunk_rows;
}

// ---- chunks: WAVES waves of 32 rows, 64 keys at a time through two buffers
template <bool BF, int D, int WAVES>
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
  const bool single = kr.hi - kr.lo <= a.chunk_split;
  const int32_t lo = kr.lo + z * a.chunk_split;
  if (z > 0 && lo >= kr.hi) return;
  const int32_t hi = min(kr.hi, lo + a.chunk_split);
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
      page[i] = __ldg(table + (min(j0 + lrow[i], hi - 1) >> a.c.page_shift));
  };
  const uint32_t k_to = lds_address(kt[0] + wave * LD * RW * D),
                 v_to = lds_address(vt[0] + wave * LD * RW * D);
  auto issue = [&](int32_t j0, int buf) {
    // all ids are waited for here: a wait between the loads would be for those loads too
#pragma unroll
    for (int i = 0; i < LD; ++i) asm volatile("" : "+v"(page[i]));
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const uint64_t at = 2 * row_at(a.c, page[i], min(j0 + lrow[i], hi - 1), lcol[i], code);
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
    if (j0 + 63 > pos_lo || j0 + 64 > hi || j0 <= win_hi) {
      hidden = true;
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int32_t j = j0 + c * 32 + 8 * (i >> 2) + 4 * h2 + (i & 3);
          if (j > pos || j >= hi || (a.window && j <= pos - a.window)) sc[c][i] = -INFINITY;
        }
    }
    float top = sc[0][0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, sc[0][i]);
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[1][i]);
    const float m2 = fmaxf(m, max_of_halves(top));
    if (__any((m2 - m) * a.c2 > kSlack)) {
      const float f = m == -INFINITY ? 0.f : exp2_fast((m - m2) * a.c2);
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
        a.lse[int64_t(q0 + tok) * a.n_heads + h] = log_sum<BF>(m, l, a.c2);
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
  if (!again || !(broken_values<BF, D>(a, table, head, max(lo, pos_lo + 1), hi) ||
                  (a.window && broken_values<BF, D>(a, table, head, lo, min(hi, win_hi + 1)))))
    return;
  wait_own<0>();  // what was stored above comes first
#pragma unroll 1
  for (; again; again &= again - 1) {
    const int r = r0 + wave * 32 + __builtin_ctzll(again), t = r / G, hh = hk * G + (r - t * G);
    put_row_by_key<BF, D>(a, table, head, q0 + t, hh, kv - n + t, lo, hi, single, a.chunk_o,
                          a.chunk_ml, (int64_t(z) * a.rows + q0 + t) * a.n_heads + hh);
  }
}

template <bool BF, int D, int NT, int WAVES>
__global__ void __launch_bounds__(WAVES * 64) k_attn_few(AttnArgs a) {
  __shared__ __align__(16) short lds[WAVES * 64 * D];
  attn_few<BF, D, NT, WAVES>(a, blockIdx.x, lds);
}
template <bool BF, int D, int WAVES>
__global__ void __launch_bounds__(WAVES * 64, 2) k_attn_chunk(AttnArgs a) {
  __shared__ __align__(16) short lds[256 * D];
  attn_chunk<BF, D, WAVES>(a, blockIdx.x, blockIdx.y, lds);
}
// Both kinds of requests in one launch: the single tokens' loads fill what the chunks' last
// work-groups leave of the card.  (24 requests of up to 8,192 tokens, 16 heads of 64, a window
// of 3,000: 82 us, 99 one after the other, 102 with the chunks last; 24 of up to 16,000, most
// of them chunks of 400 or less: 216 us, 232 one after the other, 301 with the chunks last,
// 275 with the two evenly mixed.)
template <bool BF, int D, int NT>
__global__ void __launch_bounds__(256, 2) k_attn_mixed(AttnArgs a, int chunk, int tiles) {
  __shared__ __align__(16) short lds[256 * D];
  const int block = blockIdx.x;
  if (block < chunk)
    attn_chunk<BF, D, 4>(a, block % tiles, block / tiles, lds);
  else
    attn_few<BF, D, NT, 4>(a, block - chunk, lds);
}

// ---- the splits of a row and head, joined in split order by 16-byte columns.
// A row's splits, `step` rows apart from idx0 on.
struct Parts {
  const float *o, *ml;
  int64_t idx0, step;
  int splits;
};
// Adds every PER-th split from `first` on to the four columns of `acc`.
template <int D, int PER>
__device__ inline void add_splits(const AttnArgs &a, const Parts &p, int first, int c, float top,
                                  f32x4 &acc, float &sum) {
#pragma unroll 4
  for (int i = first; i < p.splits; i += PER) {
    const int64_t idx = p.idx0 + i * p.step;
    const float mi = p.ml[idx * 2];
    const float f = part_factor(mi, top, a.c2);
    sum += f * p.ml[idx * 2 + 1];
    acc += f * *reinterpret_cast<const f32x4 *>(p.o + idx * D + c * 4);
  }
}
// The largest of the splits' maxima, by LANES neighbouring lanes.
template <int LANES>
__device__ inline float top_of(const Parts &p) {
  float top = -INFINITY;
  for (int i = threadIdx.x % LANES; i < p.splits; i += LANES)
    top = fmaxf(top, p.ml[(p.idx0 + i * p.step) * 2]);
#pragma unroll
  for (int w = LANES / 2; w; w >>= 1) top = fmaxf(top, __shfl_xor(top, w, 64));
  return top;
}
template <bool BF, int D>
__device__ inline void put_joined(const AttnArgs &a, int64_t t, int32_t h, int c, f32x4 acc,
                                  float sum, float top) {
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
  s16x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = to_16<BF>(acc[i] * inv);
  *reinterpret_cast<s16x4 *>(a.out + t * a.out_stride + h * D + c * 4) = v;
  if (c == 0 && a.lse) a.lse[t * a.n_heads + h] = log_sum<BF>(top, sum, a.c2);
}

// Few rows, often many splits: a work-group for a row and head, the splits side by side.
template <bool BF, int D>
__global__ void __launch_bounds__(256) k_attn_join_few(AttnArgs a) {
  constexpr int PER = 256 / (D / 4);  // splits side by side
  __shared__ f32x4 part[PER][D / 4];
  __shared__ float ls[PER];
  const int32_t h = blockIdx.x, s = blockIdx.y, tok = blockIdx.z;
  const int32_t q0 = __ldg(a.q_off + s), n = __ldg(a.q_off + s + 1) - q0;
  if (tok >= n || n * a.group > kFewRows) return;
  int32_t code = 0;
  const int32_t kv = checked_len(a.kv_len, s, a.max_kv, code);
  const KeyRange kr = key_range(a, n, kv, 0, n - 1);
  const int32_t len = kr.hi - kr.lo;
  if (len <= a.few_split) return;  // written whole
  const Parts p{a.few_o, a.few_ml, (int64_t(s) * a.few_tokens + tok) * a.n_heads + h,
                int64_t(a.n_seqs) * a.few_tokens * a.n_heads,
                (len + a.few_split - 1) / a.few_split};
  const float top = top_of<64>(p);
  const int g = threadIdx.x / (D / 4), c = threadIdx.x % (D / 4);
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float sum = 0.f;
  add_splits<D, PER>(a, p, g, c, top, acc, sum);
  part[g][c] = acc;
  if (c == 0) ls[g] = sum;
  __syncthreads();
  if (g) return;
  sum = 0.f;
  acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < PER; ++i) acc += part[i][c], sum += ls[i];
  put_joined<BF, D>(a, q0 + tok, h, c, acc, sum, top);
}

// Many rows, few splits: D / 4 lanes for a row and head.  (1,000 tokens of 32 heads in 2
// splits, head_dim 128: 10.8 us; with a work-group for each row and head 43.)  A wave holds
// several items, whose rows may belong to several requests.
template <bool BF, int D>
__global__ void __launch_bounds__(256) k_attn_join_chunk(AttnArgs a) {
  constexpr int LANES = D / 4;
  const int32_t it = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (it >= a.rows * a.n_heads) return;
  const int32_t t = it / a.n_heads, h = it - t * a.n_heads, c = threadIdx.x % LANES;
  const int32_t s = seq_of_own_row(a.q_off, a.n_seqs, t);
  const int32_t q0 = __ldg(a.q_off + s), n = __ldg(a.q_off + s + 1) - q0;
  if (n * a.group <= kFewRows) return;
  int32_t code = 0;
  const int32_t kv = checked_len(a.kv_len, s, a.max_kv, code);
  const int32_t r0 = ((t - q0) * a.group + h % a.group) / a.chunk_rows * a.chunk_rows;
  const KeyRange kr = key_range(a, n, kv, r0 / a.group,
                                (min(r0 + a.chunk_rows, n * a.group) - 1) / a.group);
  const int32_t len = kr.hi - kr.lo;
  if (len <= a.chunk_split) return;  // written whole
  const Parts p{a.chunk_o, a.chunk_ml, it, int64_t(a.rows) * a.n_heads,
                (len + a.chunk_split - 1) / a.chunk_split};
  const float top = top_of<LANES>(p);
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float sum = 0.f;
  add_splits<D, 1>(a, p, 0, c, top, acc, sum);
  put_joined<BF, D>(a, t, h, c, acc, sum, top);
}

// How a call's work is split: from the step's shape and the bound on lengths alone.
struct Plan {
  int32_t few_seqs, few_rows, few_tokens, few_waves, few_split, few_splits;
  int32_t chunk_seqs, chunk_rows, chunk_tiles, chunk_split, chunk_splits;
};

// A window that no length can fill is none (and positions less a window stay in 32 bits).
int32_t limited(int32_t window, const fs_step *s) { return window >= s->max_kv ? 0 : window; }

Plan plan(const fs_step *s, const fs_kv_cache *c, int32_t n_heads, int32_t window) {
  window = limited(window, s);
  Plan p = {};
  const int32_t G = n_heads / c->n_kv_heads;
  int32_t most = 0;
  for (int32_t i = 0; i < s->n_seqs; ++i) {
    const int32_t n = s->q_off_h[i + 1] - s->q_off_h[i];
    if (n == 0) continue;
    if (int64_t(n) * G <= kFewRows) {
      ++p.few_seqs;
      p.few_tokens = n > p.few_tokens ? n : p.few_tokens;
    } else {
      ++p.chunk_seqs;
      most = n > most ? n : most;
    }
  }
  p.few_rows = p.few_tokens * G;
  auto keys = [&](int32_t tokens) {  // most keys that a tile of rows sees
    const int64_t k = window ? int64_t(window) + tokens : s->max_kv;
    return int32_t(k < s->max_kv ? k : s->max_kv);
  };
  auto split_of = [&](int64_t blocks, int32_t len, int32_t want, int32_t least, int32_t most,
                      int64_t rows, int32_t &split, int32_t &splits) {
    const int64_t bytes = rows * n_heads * (c->head_dim + 2) * 4;  // of one split
    int64_t most_splits = kMostPartial / bytes;
    most_splits = most_splits < 4 ? 4 : most_splits > 512 ? 512 : most_splits;
    int64_t each = (int64_t(len) * blocks + want - 1) / want;
    each = (each + 127) / 128 * 128;
    each = each < least ? least : each > most ? most : each;
    // no more splits than their partial results may take, whatever the bound on lengths
    const int64_t few = (int64_t(len) + most_splits - 1) / most_splits;
    if (each < few) each = (few + 127) / 128 * 128;
    split = int32_t(each);
    splits = len > split ? (len + split - 1) / split : 1;
  };
  // few rows: 1,024 work-groups wanted, of 512 to 1,024 keys (4 requests of up to 500 keys,
  // 8 heads: 9.7 us whole, 13.0 in two splits of 256, and 3,000 keys 15.5 and 14.1; 64 of up
  // to 16,384: 121 us with 1,024 keys at most, 125 with 512, 127 with 2,048; one of 200,001
  // over 4 heads: 86 us, 94 with 2,048 work-groups, 90 with 512)
  p.few_waves = 4;
  if (p.few_seqs > 0) {
    const int64_t blocks = int64_t(p.few_seqs) * c->n_kv_heads;
    const int32_t len = keys(p.few_tokens);
    split_of(blocks, len, 1024, 512, 1024, int64_t(s->n_seqs) * p.few_tokens, p.few_split,
             p.few_splits);
    // Up to 1,024 keys (2,048 of head_dim 64) with a compute unit for each work-group: eight
    // waves and no join.  (4 requests, 8 heads of 128: 500 keys 8.9 us, 9.8 with four waves;
    // 1,000 keys 11.5 and, in two splits, 13.5; 30 requests of 1,000 13.4 and 17.1; 1,500 keys
    // whole 14.5, in splits 13.8.  Of 64: 1,400 keys 10.3 and 13.2, 2,000 12.9 and 14.1.)
    const int32_t whole = 131072 / c->head_dim;
    if (p.chunk_seqs == 0 && p.few_rows <= 32 && len <= whole && blocks <= 256) {
      p.few_waves = 8;
      p.few_split = whole;
      p.few_splits = 1;
    }
  }
  if (p.chunk_seqs > 0) {
    auto tiles = [&](int32_t rows) {
      return int32_t(int64_t(s->q_off_h[s->n_seqs]) * G / rows + s->n_seqs);
    };
    // 256 rows share each key tile where that still gives every compute unit a work-group
    // (head_dim 128: 4,096 rows over 32,768 keys 2.03 ms with 128 rows, 1.89 ms with 256; the
    // lighter tiles of head_dim 64 gain more from four work-groups a unit, 145 against 109 us)
    // and no request of few rows is there to run beside them (100 requests, chunks of up to
    // 300 of 8 x 4 heads and single tokens: 466 us with 256 rows, 356 with 128 and one launch;
    // chunks of up to 4,000 over 20,000 keys: 2.23 ms and 2.30)
    p.chunk_rows = c->head_dim == 128 && p.few_seqs == 0 &&
                           int64_t(tiles(256)) * c->n_kv_heads >= 256
                       ? 256
                       : 128;
    p.chunk_tiles = tiles(p.chunk_rows);
    // 512 work-groups wanted, of at least 1,024 keys (300 rows over 20,000 keys: 134 us, 154
    // with 256 work-groups, 144 with 1,024)
    const int32_t toks = p.chunk_rows / G + 2;
    split_of(int64_t(p.chunk_tiles) * c->n_kv_heads, keys(most < toks ? most : toks), 512, 1024,
             1 << 30, s->q_off_h[s->n_seqs], p.chunk_split, p.chunk_splits);
  }
  return p;
}

size_t round256(size_t x) { return (x + 255) / 256 * 256; }

// Bytes of the partial results: [rows][D] and [rows][2] floats of each kind.
struct Space {
  size_t few_o, few_ml, chunk_o, chunk_ml;
  size_t total() const { return few_o + few_ml + chunk_o + chunk_ml; }
};
Space space(const Plan &p, const fs_step *s, const fs_kv_cache *c, int32_t n_heads) {
  Space w = {};
  if (p.few_splits > 1) {
    const size_t r = size_t(p.few_splits) * s->n_seqs * p.few_tokens * n_heads;
    w.few_o = round256(r * c->head_dim * 4);
    w.few_ml = round256(r * 8);
  }
  if (p.chunk_splits > 1) {
    const size_t r = size_t(p.chunk_splits) * s->q_off_h[s->n_seqs] * n_heads;
    w.chunk_o = round256(r * c->head_dim * 4);
    w.chunk_ml = round256(r * 8);
  }
  return w;
}

template <bool BF, int D>
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
        hipLaunchKernelGGL((k_attn_mixed<BF, D, NT>), dim3(chunk + few), block, 0, stream, a, chunk,
                           tiles);
    if constexpr (NT <= 2)
      if (p.few_waves == 8)
        hipLaunchKernelGGL((k_attn_few<BF, D, NT, 8>), dim3(few), dim3(512), 0, stream, a);
    if (few > 0 && !mixed && p.few_waves == 4)
      hipLaunchKernelGGL((k_attn_few<BF, D, NT, 4>), dim3(few), block, 0, stream, a);
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
        hipLaunchKernelGGL((k_attn_chunk<BF, D, 8>), grid, dim3(512), 0, stream, a);
    if (p.chunk_rows == 128)
      hipLaunchKernelGGL((k_attn_chunk<BF, D, 4>), grid, block, 0, stream, a);
  }
  if (p.few_splits > 1)
    hipLaunchKernelGGL((k_attn_join_few<BF, D>), dim3(a.n_heads, a.n_seqs, p.few_tokens), block, 0,
                       stream, a);
  if (p.chunk_splits > 1) {
    const int64_t lanes = int64_t(a.rows) * a.n_heads * (D / 4);
    hipLaunchKernelGGL((k_attn_join_chunk<BF, D>), dim3((lanes + 255) / 256), block, 0, stream, a);
  }
}

}  // namespace

size_t attention_workspace_bytes(const fs_step *s, const fs_kv_cache *c, int32_t n_heads,
                                 int32_t window) {
  return space(plan(s, c, n_heads, window), s, c, n_heads).total();
}

hipError_t launch_attention(const fs_step *s, const fs_kv_cache *c, int32_t n_heads, float scale,
                            int32_t window, const void *q, int64_t q_stride, void *out,
                            int64_t out_stride, float *lse, void *ws, int32_t *err,
                            hipStream_t stream) {
  const Plan p = plan(s, c, n_heads, window);
  const Space w = space(p, s, c, n_heads);
  AttnArgs a;
  a.q_off = s->q_off;
  a.kv_len = s->kv_len;
  a.n_seqs = s->n_seqs;
  a.max_kv = s->max_kv;
  a.rows = s->q_off_h[s->n_seqs];
  a.n_heads = n_heads;
  a.window = limited(window, s);
  a.group = n_heads / c->n_kv_heads;
  a.c = dev_cache(c);
  a.q = static_cast<const short *>(q);
  a.out = static_cast<short *>(out);
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.lse = lse;
  // a scale of 0 makes every visible score equal; a factor of 0 would turn -inf into NaN
  const float c2 = (scale < 0.f ? -scale : scale) * 1.44269504088896341f;
  a.c2 = c2 > 1.2e-38f ? c2 : 1.2e-38f;
  a.flip = scale < 0.f;
  a.few_split = p.few_split;
  a.few_tokens = p.few_tokens;
  a.chunk_rows = p.chunk_rows;
  a.chunk_split = p.chunk_split;
  char *at = static_cast<char *>(ws);
  a.few_o = reinterpret_cast<float *>(at);
  a.few_ml = reinterpret_cast<float *>(at + w.few_o);
  a.chunk_o = reinterpret_cast<float *>(at + w.few_o + w.few_ml);
  a.chunk_ml = reinterpret_cast<float *>(at + w.few_o + w.few_ml + w.chunk_o);
  a.err = err;
  const bool bf = c->dtype == FS_BF16;
  if (bf && c->head_dim == 128)
    run<true, 128>(a, p, stream);
  else if (bf)
    run<true, 64>(a, p, stream);
  else if (c->head_dim == 128)
    run<false, 128>(a, p, stream);
  else
    run<false, 64>(a, p, stream);
  return hipGetLastError();
}

}  // namespace fs
