// Attention of the step's rows over a paged cache held in 4 bits:
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q . k_j - m),  over the keys a row sees,
// with the softmax's running reference, the split of the work and the joins of the kernels over
// the 16-bit cache, and codes in place of values.  A group of 32 values and its scale become
// 16-bit values exactly (one conversion instruction for two of them).
//   k_attn4_few    requests of at most 64 rows: bound by the cache's bytes where many are long
//                  (64 of 16,384 tokens: 219 to 227 us, 5.0 to 5.2 TB/s; 128 of up to 16,384,
//                  229,312 in all, 70 us, 3.6 TB/s, 61 and 4.1 without the join and the launch), by
//                  the chain from lengths to pages to keys where few are (4 of 500: 9.0 us).  K
//                  feeds the first product from registers: the sum over a head's dimensions may be
//                  taken in any order, so each lane takes 32 (or 16) neighbouring ones of a key, 16
//                  bytes of codes with one scale, and a wave's load is 16 whole keys without a gap.
//                  V is wanted with keys along a lane, while its codes and scales lie along
//                  dimensions: it goes through LDS as 16-bit values and is read back transposed.
//   k_attn4_chunk  larger chunks: bound by the chain of a tile's steps (scores, exponentials,
//                  products) at two waves a SIMD (4,096 rows over 32,768 keys 1.84 to 1.96 ms from
//                  card to card, 1.05 to 1.12 PFLOP/s; in half precision 1.88 to 2.01; head_dim 64
//                  1.25, 0.82 PFLOP/s).  K and V go through LDS as 16-bit values.
//   k_attn4_mixed  both in one launch; the joins are those of the 16-bit cache, or
//   k_attn4_join_many for few rows in very many splits.
#include <type_traits>

#include "fs_attn.h"
#include "fs_cache.h"

namespace fs {

namespace {

struct Attn4Args : AttnArgs {  // `c` is the cache's codes, in bytes
  DevScales sc;
};

// The units of the exponentials (fs_attn.h).  Scales reach 2^125 for bfloat16: with 2^-18 the
// sums of 1,000 such values stay in fp32's range, and values down to 2^-100 above its smallest.
template <bool BF>
constexpr float kLift4 = BF ? -18.f : 7.f;

// The most that a lane's 32 probabilities of a tile may sum to before its reference is moved: 2^14
// times the reference's own for bfloat16, and 2^8 times for half precision, below its 65,504.
template <bool BF>
constexpr float kMostSum = BF ? 0x1p-4f : 0x1p15f;

// A quarter of the 16-bit cache's bytes: twice its longest splits (64 requests of 16,384 tokens:
// 219 us, 233 with 1,024 keys) and whole requests (30 of 2,000 tokens: 19.4 us, 23.3 in splits; 8
// of 1,100 11.7 and 15.0; 4 of 2,000 16.6 and 15.7).  (Finer splits, 4,096 work-groups wanted,
// help a few requests of which one is long, 9 of 2 to 18,596 tokens 27 us and 45, and cost those
// that are alike, 32 of 8,000 46 and 41, 8 of 32,768 51 and 44.)
constexpr int32_t kFewMost4 = 2048;
constexpr int32_t kFewWhole4 = 262144;
constexpr int32_t kOnce4 = 2048;
// Splits go by the bound on lengths, and chunks of several requests seldom all reach it: twice the
// work-groups.  (4 chunks of 300 rows over 20,000, 3,000, 1,000 and 500 keys: 245 us, 342 with 512
// work-groups, all over 20,000 492 and 527; 8 of 100 over 100 to 8,000, head_dim 64: 40 and 67, all
// over 8,000 67 and 94; but 3 of 1,000 over 9,000 488 and 462, 16 of 64 over 4,000 108 and 94.)
constexpr int32_t kChunkWant4 = 1024;
// (100 rows over 4,000 keys 31.2 us, 38.8 in splits of 1,024 keys, 33.4 of 256; 255 rows over
// 11,191, head_dim 64, 31.9, 37.2 and 31.6; 300 over 20,000 take longer splits.)
constexpr int32_t kChunkLeast4 = 512;

// Codes of N neighbouring values: 16 bytes for 32 of them, 8 for 16.
template <int N>
using Codes = uint32_t __attribute__((ext_vector_type(N / 8)));

// A group that counts as NaN is multiplied as zeros; the rows that see such a key get NaN in
// the group's columns at the end: bit g of `poison` for the columns 32 g .. .
template <int N, class Acc>
__device__ inline void put_poison(uint32_t poison, int group, Acc &o) {
  if (poison >> group & 1)
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = NAN;
}

// Tiles of 16-bit values: key rows further apart than their D values, so that 16 rows' chunks,
// and 4 rows' transposed reads, fall on different banks at addresses that differ by constants
// (places swapped by row, as over the 16-bit cache, take a register for each address).
template <int D>
constexpr int kRow = D == 128 ? 144 : 72;
template <int D, int KEYS>
constexpr int kTile = KEYS * kRow<D> + 8;
template <int D>
__device__ inline int tile_row(int r) {
  return r * kRow<D> + (D == 128 ? (r >> 3 & 1) * 8 : 0);
}

// ---- few rows: NT tiles of 16 rows, WAVES waves, which take 32 keys each in turn
template <bool BF, int D, int NT, int WAVES>
__device__ __forceinline__ void attn4_few(const Attn4Args &a, int block, short *lds) {
  constexpr int KS = D / 32;  // matrix steps of a score
  constexpr int DB = D / 16;  // 16-column blocks of an output row
  constexpr int DL = D / 4;   // neighbouring dimensions of a key that a lane takes
  constexpr int kIds = 512;   // page ids kept in LDS
  constexpr bool kTwoParts = NT <= 2;  // of a probability
  constexpr int VB = 4;       // 16-column blocks of V read at once
  __shared__ float wm[WAVES][NT * 16], wl[WAVES][NT * 16];
  __shared__ uint32_t ids[kIds];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, g4 = lane >> 4;
  // (heads fastest, and each split shifts the requests by one: see the 16-bit kernel)
  const int hk = block % a.c.n_kv_heads, sz = block / a.c.n_kv_heads;
  const int z = sz / a.n_seqs, s = (sz + z) % a.n_seqs;
  const int32_t q0 = __ldg(a.q_off + s), n = __ldg(a.q_off + s + 1) - q0;
  const int G = a.group, R = n * G;
  if (R <= 0 || R > kFewRows) return;
  int32_t code = 0;
  const int32_t kv = checked_len(a.kv_len, s, a.max_kv, code);
  const KeyRange kr = key_range(a, n, kv, 0, n - 1);
  const bool single = kr.length() <= a.few_split;
  const int32_t lo = z * a.few_split;
  if (z > 0 && lo >= kr.length()) return;
  const int32_t hi = min(kr.length(), lo + a.few_split);
  const int32_t *table = a.c.table + s * a.c.table_stride;
  // where this lane's part of a key row begins
  const uint32_t inside = hk * a.c.head_stride + g4 * (DL / 2);
  const uint32_t s_inside = hk * a.sc.head_stride + g4 * DL / 32;

  // queries: row r16 of each tile, 8 of this lane's dimensions at each step
  s16x8 qf[NT][KS];
  int32_t pos[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    // (rows past the last are that one again)
    const int r = min(t * 16 + r16, R - 1), tok = r / G, h = hk * G + (r - tok * G);
    pos[t] = kv - n + tok;
    const short *qp = a.q + (q0 + tok) * a.q_stride + h * D + g4 * DL;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      qf[t][k] = *reinterpret_cast<const s16x8 *>(qp + k * 8);
      if (a.flip) qf[t][k] ^= short(0x8000);
    }
  }
  f32x4 o[NT][DB] = {};
  float m[NT], l[NT];
  uint32_t poison[NT] = {};
#pragma unroll
  for (int t = 0; t < NT; ++t) m[t] = -INFINITY, l[t] = 0.f;

  short *const v_to = lds + wave * kTile<D, 32> + tile_row<D>(r16) + g4 * DL;
  const short *const v_from =
      lds + wave * kTile<D, 32> + tile_row<D>(4 * g4 + (r16 >> 2)) + (r16 & 3) * 4;

  for (int32_t from = lo; from < hi;) {
    const PageIds span = page_ids<true>(kr, from, hi, a.c.page_shift, kIds);
    const int32_t end = span.end;
    __syncthreads();
    for (int i = tid; i < span.n; i += WAVES * 64) {
      const uint32_t page = __ldg(table + span.page(i));
      if (page >= a.c.n_pages) code = FS_E_RANGE;
      ids[i] = page < a.c.n_pages ? page : 0;
    }
    __syncthreads();
    const int32_t first = from + wave * 32;
    const int32_t tiles = first < end ? (end - first + WAVES * 32 - 1) / (WAVES * 32) : 0;
    // this lane's part of two keys
    Codes<DL> kc[2], vc[2];
    uint32_t ks[2], vs[2];
    auto load = [&](int32_t t) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int32_t j = kr.key(min(first + t * (WAVES * 32) + b * 16 + r16, end - 1));
        const uint32_t page = ids[span.slot(j)], slot = j & ((1 << a.c.page_shift) - 1);
        const uint64_t at =
            uint64_t(page) * a.c.page_stride + (inside + slot * a.c.token_stride);
        const uint64_t sat =
            uint64_t(page) * a.sc.page_stride + (s_inside + slot * a.sc.token_stride);
        kc[b] = *reinterpret_cast<const Codes<DL> *>(a.c.k + at);
        vc[b] = *reinterpret_cast<const Codes<DL> *>(a.c.v + at);
        ks[b] = a.sc.k[sat];
        vs[b] = a.sc.v[sat];
      }
    };
    if (tiles > 0) load(0);
    for (int32_t t = 0; t < tiles; ++t) {
      const int32_t j0 = first + t * (WAVES * 32);
      f32x4 sc[NT][2] = {};
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const float unit = scale_of<BF>(ks[b]);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const s16x8 kf = values8<BF>(kc[b][k], unit);
#pragma unroll
          for (int r = 0; r < NT; ++r) sc[r][b] = mfma_16x16x32<BF>(kf, qf[r][k], sc[r][b]);
        }
      }
      // V: this lane's dimensions of two keys, as chunks of 8
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const float unit = scale_of<BF>(vs[b]);
        const bool bad = vs[b] > kTopScale<BF>;
#pragma unroll
        for (int k = 0; k < KS; ++k)
          *reinterpret_cast<s16x8 *>(v_to + b * 16 * kRow<D> + k * 8) =
              values8<BF>(bad ? 0 : vc[b][k], unit);
      }
      if (__any(max(max(ks[0], ks[1]), max(vs[0], vs[1])) > kTopScale<BF>)) {
#pragma unroll 1
        for (int b = 0; b < 2; ++b) {
          uint64_t bad = __ballot((b ? ks[1] : ks[0]) > kTopScale<BF>);
          bad |= bad >> 32;
          bad |= bad >> 16;  // bit i: key i of the 16
#pragma unroll
          for (int r = 0; r < NT; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (bad >> (g4 * 4 + i) & 1) (b ? sc[r][1] : sc[r][0])[i] = NAN;
          for (uint64_t vbad = __ballot((b ? vs[1] : vs[0]) > kTopScale<BF>); vbad;
               vbad &= vbad - 1) {
            const int i = __builtin_ctzll(vbad);
            const int32_t v = j0 + b * 16 + (i & 15), j = kr.key(v);
#pragma unroll
            for (int r = 0; r < NT; ++r)
              if (j <= pos[r] && v < end &&
                  (a.window == 0 || j > pos[r] - a.window || j < a.sinks))
                poison[r] |= 1u << ((i >> 4) * DL / 32);
          }
        }
      }
      // the codes have been used: the next ones come while the rest is computed
      if (t + 1 < tiles) load(t + 1);
      const int32_t key0 = kr.key(j0), key31 = kr.key(j0 + 31);
      // keys that some row does not see
      const bool edge = j0 + 32 > end || key31 > kv - n || (a.window && key0 <= kv - 1 - a.window);
      s16x8 pf[NT], pl[NT];
#pragma unroll
      for (int r = 0; r < NT; ++r) {
        float p[8], top = -INFINITY;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) p[b * 4 + i] = sc[r][b][i];
        if (edge) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int32_t v = j0 + b * 16 + g4 * 4 + i, j = kr.key(v);
              const bool see = j <= pos[r] && v < end &&
                               (a.window == 0 || j > pos[r] - a.window || j < a.sinks);
              if (!see) p[b * 4 + i] = -INFINITY;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, p[i]);
        top = max_of_halves(max_of_16s(top));
        // a row's reference moves by its own scores alone (-inf less -inf is no number and asks for
        // nothing)
        const float m2 = (top - m[r]) * a.c2 > kSlack ? top : m[r];
        if (__any(m2 != m[r])) {
          const float f = m[r] == -INFINITY ? 0.f : part_factor(m[r], m2, a.c2);
          l[r] *= f;
#pragma unroll
          for (int d = 0; d < DB; ++d) o[r][d] *= f;
          m[r] = m2;
        }
        const float mc = reference(m[r], a.c2) - kLift4<BF>;
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
      for (int d0 = 0; d0 < DB; d0 += VB) {
        s16x8 vv[VB];
#pragma unroll
        for (int d = 0; d < VB; ++d)
          vv[d] = __builtin_shufflevector(read_tr(v_from + (d0 + d) * 16),
                                          read_tr(v_from + 16 * kRow<D> + (d0 + d) * 16), 0, 1, 2,
                                          3, 4, 5, 6, 7);
#pragma unroll
        for (int r = 0; r < NT; ++r) {
#pragma unroll
          for (int d = 0; d < VB; ++d) o[r][d0 + d] = mfma_16x16x32<BF>(vv[d], pf[r], o[r][d0 + d]);
          if (kTwoParts)
#pragma unroll
            for (int d = 0; d < VB; ++d)
              o[r][d0 + d] = mfma_16x16x32<BF>(vv[d], pl[r], o[r][d0 + d]);
        }
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
    if (__any(poison[t] != 0))
#pragma unroll
      for (int d = 0; d < DB; ++d) put_poison<4>(poison[t], d / 2, o[t][d]);
  }
  float *buf = reinterpret_cast<float *>(lds);  // [WAVES][16][D / 2]: half of the columns
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
            a.lse[int64_t(q0 + tok) * a.n_heads + h] = log_sum(top, sum, a.c2, kLift4<BF>);
        } else {
          const int64_t idx =
              ((int64_t(z) * a.n_seqs + s) * a.few_tokens + tok) * a.n_heads + h;
          *reinterpret_cast<f32x4 *>(a.few_o + idx * D + cc) = acc;
          if (cc == 0) a.few_ml[idx * 2] = top, a.few_ml[idx * 2 + 1] = sum;
        }
      }
    }
  }
}

// ---- chunks: WAVES waves of 32 rows, 64 keys at a time through two buffers of 16-bit values
template <bool BF, int D, int WAVES>
__device__ __forceinline__ void attn4_chunk(const Attn4Args &a, int block, int z, short *lds) {
  __shared__ __align__(16) uint8_t sb[2][2][64 * (D / 32)];  // the scale bytes of K's and V's tiles
  __shared__ int odd;                          // whether one of them counts as NaN
  constexpr int KS = D / 16;       // matrix steps of a score
  constexpr int DB = D / 32;       // 32-column blocks of an output row: groups
  constexpr int RW = 64 / DB;      // keys of a wave's load: a lane takes a group of one key
  constexpr int LD = 2 * 64 / RW / WAVES;  // a wave's loads of K and V for 64 keys
  static_assert(LD >= 1, "a wave loads whole rows");
  // K's two buffers, then V's, as 16-bit values.  (The matrix cores' products of 4-bit numbers
  // would take K's codes as they are, with the queries as two 8-bit parts, in 1,657 us for 4,096
  // rows over 32,768 keys; but they drop what lies 2^-14 below the largest of the products that
  // they add at once, and scores are sums of 32 bits.)
  constexpr int VT = 2 * kTile<D, 64>;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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
  const bool single = kr.length() <= a.chunk_split;
  const int32_t lo = z * a.chunk_split;
  if (z > 0 && lo >= kr.length()) return;
  const int32_t hi = min(kr.length(), lo + a.chunk_split);
  const int32_t *table = a.c.table + s * a.c.table_stride;

  const int row = r0 + wave * 32 + r32;
  const int tok = min(row, R - 1) / G, h = hk * G + (min(row, R - 1) - tok * G);
  const int32_t pos = kv - n + tok;
  // the wave's first row, and the first key that its last row's window leaves
  const int32_t pos_lo = kv - n + min(r0 + wave * 32, R - 1) / G;
  const int32_t win_hi =
      a.window ? kv - n + min(r0 + wave * 32 + 31, R - 1) / G - a.window : INT32_MIN;
  s16x8 qf[KS];
  const short *qp = a.q + (q0 + tok) * a.q_stride + h * D + h2 * 8;
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    qf[k] = *reinterpret_cast<const s16x8 *>(qp + k * 16);
    if (a.flip) qf[k] ^= short(0x8000);
  }
  f32x16 o[DB] = {};
  float m = -INFINITY, mc = 0.f, l = 0.f;
  uint32_t poison = 0;

  // Load i of the wave: 64 / DB keys' K (then V) rows, the keys along the lanes, so that 16
  // lanes write 16 rows of a tile (and no two of them the same banks).
  const int group = lane / RW;
  int32_t lrow[LD];
  uint32_t page[LD];
  bool val[LD];
#pragma unroll
  for (int i = 0; i < LD; ++i) {
    const int u = i * WAVES + wave;
    val[i] = u >= 64 / RW;
    lrow[i] = (val[i] ? u - 64 / RW : u) * RW + lane % RW;
  }
  auto pages = [&](int32_t j0) {
#pragma unroll
    for (int i = 0; i < LD; ++i)
      page[i] = __ldg(table + (kr.key(min(j0 + lrow[i], hi - 1)) >> a.c.page_shift));
  };
  Codes<32> w[LD];
  uint32_t ws[LD];
  auto load = [&](int32_t j0) {
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int32_t j = kr.key(min(j0 + lrow[i], hi - 1));
      uint32_t id = page[i];
      if (id >= a.c.n_pages) {
        code = FS_E_RANGE;
        id = 0;
      }
      const uint32_t slot = j & ((1 << a.c.page_shift) - 1);
      const uint64_t at = uint64_t(id) * a.c.page_stride +
                          (hk * a.c.head_stride + group * 16 + slot * a.c.token_stride);
      const uint64_t sat = uint64_t(id) * a.sc.page_stride +
                           (hk * a.sc.head_stride + group + slot * a.sc.token_stride);
      w[i] = *reinterpret_cast<const Codes<32> *>((val[i] ? a.c.v : a.c.k) + at);
      ws[i] = (val[i] ? a.sc.v : a.sc.k)[sat];
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const bool bad = ws[i] > kTopScale<BF>;
      const float unit = scale_of<BF>(ws[i]);
      short *to = lds + (val[i] ? VT : 0) + buf * kTile<D, 64> + tile_row<D>(lrow[i]) + group * 32;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        *reinterpret_cast<s16x8 *>(to + k * 8) = values8<BF>(bad ? 0 : w[i][k], unit);
      sb[buf][val[i]][lrow[i] * DB + group] = uint8_t(ws[i]);
      if (bad) odd = 1;
    }
  };
  if (tid == 0) odd = 0;
  __syncthreads();
  if (lo < hi) {
    pages(lo);
    load(lo);
    pages(lo + 64);
    put(0);
    load(lo + 64);  // (past the end: the last key)
    pages(lo + 128);
  }
  __syncthreads();
  int buf = 0;
  for (int32_t j0 = lo; j0 < hi; j0 += 64, buf ^= 1) {
    if (j0 + 64 < hi) {
      put(buf ^ 1);
      load(j0 + 128);
      pages(j0 + 192);
    }
    f32x16 sc[2] = {};
    const short *const kb = lds + buf * kTile<D, 64> + tile_row<D>(r32) + h2 * 8;
#pragma unroll
    for (int k0 = 0; k0 < KS; k0 += 4) {
      s16x8 kf[4][2];
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int c = 0; c < 2; ++c)
          kf[k][c] = *reinterpret_cast<const s16x8 *>(kb + c * 32 * kRow<D> + (k0 + k) * 16);
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int c = 0; c < 2; ++c) sc[c] = mfma_32x32x16<BF>(kf[k][c], qf[k0 + k], sc[c]);
    }
    if (__builtin_amdgcn_readfirstlane(odd)) {
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = c * 32 + 8 * (i >> 2) + 4 * h2 + (i & 3);
#pragma unroll
          for (int g = 0; g < DB; ++g)
            if (sb[buf][0][key * DB + g] > kTopScale<BF>) sc[c][i] = NAN;
        }
#pragma unroll 1
      for (int key = 0; key < 64; ++key) {
        const int32_t v = j0 + key, j = kr.key(v);
        if (j > pos || v >= hi || (a.window && j <= pos - a.window && j >= a.sinks)) continue;
#pragma unroll
        for (int g = 0; g < DB; ++g)
          if (sb[buf][1][key * DB + g] > kTopScale<BF>) poison |= 1u << g;
      }
    }
    // keys that some row of the wave does not see
    if (kr.key(j0 + 63) > pos_lo || j0 + 64 > hi || kr.key(j0) <= win_hi) {
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int32_t v = j0 + c * 32 + 8 * (i >> 2) + 4 * h2 + (i & 3), j = kr.key(v);
          if (j > pos || v >= hi || (a.window && j <= pos - a.window && j >= a.sinks))
            sc[c][i] = -INFINITY;
        }
    }
    // Probabilities, and their sum, by the reference of the tiles before; only where a row has
    // none yet, or a sum shows that a score passes it by far, the row's maximum is looked for.
    // (Rows keep their own: what one holds does not show in another's rounding.)
    s16x8 pf[4];
    float sum;
    bool moves = m == -INFINITY;
    for (bool again = false;; again = true) {
      if (__any(moves)) {
        float top = sc[0][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, sc[0][i]);
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[1][i]);
        top = max_of_halves(top);
        const float m2 = moves ? fmaxf(m, top) : m;
        const float f = m == -INFINITY ? 0.f : part_factor(m, m2, a.c2);
        l *= f;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] *= f;
        m = m2;
        mc = reference(m, a.c2) - kLift4<BF>;
      }
      sum = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[i] = exp2_fast(fmaf(sc[u >> 1][(u & 1) * 8 + i], a.c2, -mc));
          sum += p[i];
        }
        pf[u] = pack8<BF>(p);
      }
      if (again || !__any(sum > kMostSum<BF>)) break;
      moves = max_of_halves(sum) > kMostSum<BF>;
    }
    l += sum;
    const short *const vb = lds + VT + buf * kTile<D, 64> + tile_row<D>(4 * h2 + ((lane & 15) >> 2)) +
                            (lane >> 4 & 1) * 16 + (lane & 3) * 4;
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        // keys 4 h2 .. + 3 and 8 + 4 h2 .. + 3 of the 16
        const short *from = vb + u * 16 * kRow<D> + d * 32;
        o[d] = mfma_32x32x16<BF>(__builtin_shufflevector(read_tr(from), read_tr(from + tile_row<D>(8)),
                                                         0, 1, 2, 3, 4, 5, 6, 7),
                                 pf[u], o[d]);
      }
    // (what the wave has read and written is done; loads from memory stay under way)
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  }
  raise_err(a.err, code);
  l += __shfl_xor(l, 32, 64);
  if (__any(poison != 0))
#pragma unroll
    for (int d = 0; d < DB; ++d) put_poison<16>(poison, d, o[d]);
  if (row >= R) return;
  if (single) {
    const float inv = l > 0.f ? 1.f / l : 0.f;
    short *op = a.out + (q0 + tok) * a.out_stride + h * D;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s16x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = to_16<BF>(o[d][i * 4 + e] * inv);
        *reinterpret_cast<s16x4 *>(op + d * 32 + i * 8 + h2 * 4) = v;
      }
    if (h2 == 0 && a.lse) a.lse[int64_t(q0 + tok) * a.n_heads + h] = log_sum(m, l, a.c2, kLift4<BF>);
  } else {
    const int64_t idx = (int64_t(z) * a.rows + q0 + tok) * a.n_heads + h;
    float *op = a.chunk_o + idx * D;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4 *>(op + d * 32 + i * 8 + h2 * 4) =
            f32x4{o[d][i * 4], o[d][i * 4 + 1], o[d][i * 4 + 2], o[d][i * 4 + 3]};
    if (h2 == 0) a.chunk_ml[idx * 2] = m, a.chunk_ml[idx * 2 + 1] = l;
  }
}

template <bool BF, int D, int NT, int WAVES>
__global__ void __launch_bounds__(WAVES * 64, NT == 1 ? 4 : NT == 2 ? (D == 64 ? 3 : 2) : D == 64 ? 2 : 1)
k_attn4_few(Attn4Args a) {
  __shared__ __align__(16) short lds[WAVES * kTile<D, 32>];
  attn4_few<BF, D, NT, WAVES>(a, blockIdx.x, lds);
}
template <bool BF, int D, int WAVES>
__global__ void __launch_bounds__(WAVES * 64, 2) k_attn4_chunk(Attn4Args a) {
  __shared__ __align__(16) short lds[4 * kTile<D, 64>];
  attn4_chunk<BF, D, WAVES>(a, blockIdx.x, blockIdx.y, lds);
}
// Both kinds of requests in one launch, as over the 16-bit cache.
template <bool BF, int D, int NT>
__global__ void __launch_bounds__(256, 2) k_attn4_mixed(Attn4Args a, int chunk, int tiles) {
  __shared__ __align__(16) short lds[4 * kTile<D, 64>];
  const int block = blockIdx.x;
  if (block < chunk)
    attn4_chunk<BF, D, 4>(a, block % tiles, block / tiles, lds);
  else
    attn4_few<BF, D, NT, 4>(a, block - chunk, lds);
}

// The join of few rows in very many splits: a work-group for 32 columns of a row and head, 32
// splits side by side.  (One request of 200,001 tokens, 32 heads in 224 splits: 34.5 us, 32.5 to
// 36.6 from card to card, 35.9 on the first with a work-group for a row and head; 8 of 32,768 in 64
// splits 43.8 and 43.3.)
constexpr int kManySplits = 128;
template <bool BF, int D>
__global__ void __launch_bounds__(256) k_attn4_join_many(Attn4Args a) {
  __shared__ f32x4 part[4][8];
  __shared__ float ls[4];
  const int32_t h = blockIdx.x / (D / 32), s = blockIdx.y, tok = blockIdx.z;
  const int32_t q0 = __ldg(a.q_off + s), n = __ldg(a.q_off + s + 1) - q0;
  if (tok >= n || n * a.group > kFewRows) return;
  int32_t code = 0;
  const int32_t kv = checked_len(a.kv_len, s, a.max_kv, code);
  const int32_t len = key_range(a, n, kv, 0, n - 1).length();
  if (len <= a.few_split) return;  // written whole
  const Parts p{a.few_o, a.few_ml, (int64_t(s) * a.few_tokens + tok) * a.n_heads + h,
                int64_t(a.n_seqs) * a.few_tokens * a.n_heads,
                (len + a.few_split - 1) / a.few_split};
  const float top = top_of<64>(p);
  const int tid = threadIdx.x, c = blockIdx.x % (D / 32) * 8 + tid % 8;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float sum = 0.f;
  add_splits<D, 32>(a, p, tid / 8, c, top, acc, sum);
#pragma unroll
  for (int w = 8; w < 64; w <<= 1) {
    sum += __shfl_xor(sum, w, 64);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] += __shfl_xor(acc[i], w, 64);
  }
  if ((tid & 63) < 8) part[tid >> 6][tid & 63] = acc, ls[tid >> 6] = sum;
  __syncthreads();
  if (tid >= 8) return;
  acc = part[0][tid] + part[1][tid] + part[2][tid] + part[3][tid];
  put_joined<BF, D>(a, q0 + tok, h, c, acc, ls[0] + ls[1] + ls[2] + ls[3], top);
}

template <bool BF, int D>
void run(const Attn4Args &a, const Plan &p, hipStream_t stream) {
  const dim3 block(256);
  const int few = p.few_seqs > 0 ? a.n_seqs * a.c.n_kv_heads * p.few_splits : 0;
  const int tiles = p.chunk_tiles * a.c.n_kv_heads;
  const int chunk = p.chunk_seqs > 0 ? tiles * p.chunk_splits : 0;
  // In one launch where one kernel holds both: at head_dim 128 it takes all 256 registers, and what
  // it spills, 5 of them, is stored ahead of the chunks' loop and loaded after it, as 3 are by
  // k_attn4_chunk alone.
  const bool mixed = few > 0 && chunk > 0 && p.chunk_rows == 128 && (D == 64 || p.few_rows <= 32);
  auto by_rows = [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    if constexpr (D == 64 || NT <= 2)
      if (mixed)
        hipLaunchKernelGGL((k_attn4_mixed<BF, D, NT>), dim3(chunk + few), block, 0, stream, a,
                           chunk, tiles);
    if constexpr (NT <= 2)
      if (p.few_waves == 8)
        hipLaunchKernelGGL((k_attn4_few<BF, D, NT, 8>), dim3(few), dim3(512), 0, stream, a);
    if (few > 0 && !mixed && p.few_waves == 4)
      hipLaunchKernelGGL((k_attn4_few<BF, D, NT, 4>), dim3(few), block, 0, stream, a);
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
        hipLaunchKernelGGL((k_attn4_chunk<BF, D, 8>), grid, dim3(512), 0, stream, a);
    if (p.chunk_rows == 128)
      hipLaunchKernelGGL((k_attn4_chunk<BF, D, 4>), grid, block, 0, stream, a);
  }
  if (p.few_splits >= kManySplits)
    hipLaunchKernelGGL((k_attn4_join_many<BF, D>), dim3(a.n_heads * (D / 32), a.n_seqs, p.few_tokens),
                       block, 0, stream, a);
  else if (p.few_splits > 1)
    hipLaunchKernelGGL((k_attn_join_few<BF, D>), dim3(a.n_heads, a.n_seqs, p.few_tokens), block, 0,
                       stream, a);
  if (p.chunk_splits > 1) {
    const int64_t lanes = int64_t(a.rows) * a.n_heads * (D / 4);
    hipLaunchKernelGGL((k_attn_join_chunk<BF, D>), dim3((lanes + 255) / 256), block, 0, stream, a);
  }
}

}  // namespace

size_t attention4_workspace_bytes(const fs_step *s, const fs_kv_cache4 *c, int32_t n_heads,
                                  int32_t window, int32_t sinks) {
  const Shape sh = shape_of(s, n_heads, c->n_kv_heads, c->head_dim, window, sinks, kFewMost4,
                            kFewWhole4, kOnce4, kChunkWant4, kChunkLeast4);
  return space(plan(s, sh), s, sh).total();
}

hipError_t launch_attention4(const fs_step *s, const fs_kv_cache4 *c, int32_t dtype,
                             int32_t n_heads, float scale, int32_t window, int32_t sinks,
                             const void *q, int64_t q_stride, void *out, int64_t out_stride,
                             float *lse, void *ws, int32_t *err, hipStream_t stream) {
  const Shape sh = shape_of(s, n_heads, c->n_kv_heads, c->head_dim, window, sinks, kFewMost4,
                            kFewWhole4, kOnce4, kChunkWant4, kChunkLeast4);
  const Plan p = plan(s, sh);
  Attn4Args a;
  fill_args(a, p, space(p, s, sh), sh, s, scale, q, q_stride, out, out_stride, lse, ws, err);
  a.c = dev_codes(c);
  a.sc = dev_scales(c);
  a.lift = dtype == FS_BF16 ? kLift4<true> : kLift4<false>;
  if (dtype == FS_BF16)
    c->head_dim == 128 ? run<true, 128>(a, p, stream) : run<true, 64>(a, p, stream);
  else
    c->head_dim == 128 ? run<false, 128>(a, p, stream) : run<false, 64>(a, p, stream);
  return hipGetLastError();
}

}  // namespace fs
