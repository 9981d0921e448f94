// Shared by the attention kernels over the 16-bit and the 4-bit cache (internal): the keys a
// row sees, the softmax's running reference, row tiles of chunks, the join of splits, and
// how a call's work is split.
#pragma once
#include "fs_engine.h"

namespace fs {

namespace {

constexpr int kFewRows = 64;    // rows (tokens times group) that k_attn_few takes
constexpr int64_t kMostPartial = int64_t(1) << 28;  // bytes of partial results, about
constexpr float kLn2 = 0.693147180559945309f;

struct AttnArgs {
  const int32_t *q_off, *kv_len;
  int32_t n_seqs, max_kv, rows, n_heads, window, group;
  int32_t sinks;  // first keys that a window leaves visible (0 without a window)
  DevCache c;
  const short *q;
  short *out;
  int64_t q_stride, out_stride;
  float *lse;
  float c2;            // |scale| * log2(e)
  float lift;          // the exponentials are in units of 2^-lift
  uint32_t flip;       // sign of the scale, applied to the queries
  int32_t few_split;   // keys of a split (k_attn_few)
  int32_t few_tokens;  // most tokens of a request that k_attn_few takes
  int32_t chunk_rows;  // rows of a work-group of k_attn_chunk
  int32_t chunk_split;
  float *few_o, *few_ml;      // [splits][n_seqs][few_tokens][heads][D], [..][2]
  float *chunk_o, *chunk_ml;  // [splits][rows][heads][D], [..][2]
  int32_t *err;
};

// Keys that the tokens tok0 .. tok1 of a request with n new and kv cached ones see: the first
// `sink` and lo .. hi - 1, sink <= lo.  Work is split by their places 0 .. length() - 1.
struct KeyRange {
  int32_t sink, lo, hi;
  __device__ int32_t length() const { return sink + (hi - lo); }
  __device__ int32_t key(int32_t place) const { return place < sink ? place : place + (lo - sink); }
};
__device__ inline KeyRange key_range(const AttnArgs &a, int32_t n, int32_t kv, int32_t tok0,
                                     int32_t tok1) {
  KeyRange r;
  r.lo = a.window ? max(0, kv - n + tok0 - a.window + 1) : 0;
  r.hi = max(0, kv - n + tok1 + 1);
  r.sink = min(a.sinks, r.lo);
  return r;
}

// The pages of the keys from place `from` on (at most `most` of them, before place hi): the
// first sink_pages of them hold sinks, the rest the keys from lo on.
struct PageIds {
  int32_t end;  // the place after the last key whose page is among them
  int32_t n, shift, sink, sink_p0, sink_pages, p0;
  __device__ int32_t page(int32_t i) const {
    return i < sink_pages ? sink_p0 + i : p0 + (i - sink_pages);
  }
  __device__ int32_t slot(int32_t key) const {
    const int32_t p = key >> shift;
    return key < sink ? p - sink_p0 : p - p0 + sink_pages;
  }
};
template <bool SINK>
__device__ inline PageIds page_ids(const KeyRange &kr, int32_t from, int32_t hi, int32_t shift,
                                   int32_t most) {
  PageIds s;
  s.shift = shift;
  s.sink = s.sink_p0 = s.sink_pages = 0;
  if constexpr (!SINK) {  // places are keys
    s.p0 = from >> shift;
    s.end = int32_t(min(int64_t(hi), int64_t(s.p0 + most) << shift));
    s.n = ((s.end - 1) >> shift) - s.p0 + 1;
    return s;
  } else {
    const int32_t last = kr.key(hi - 1);
    if (from >= kr.sink) {
      s.p0 = kr.key(from) >> shift;
      const int32_t end = int32_t(min(int64_t(last) + 1, int64_t(s.p0 + most) << shift));
      s.end = end - (kr.lo - kr.sink);
      s.n = ((end - 1) >> shift) - s.p0 + 1;
      return s;
    }
    s.sink = kr.sink;
    s.sink_p0 = from >> shift;
    s.p0 = kr.lo >> shift;
    s.end = int32_t(min(int64_t(min(hi, kr.sink)), int64_t(s.sink_p0 + most) << shift));
    s.sink_pages = ((s.end - 1) >> shift) - s.sink_p0 + 1;
    s.n = s.sink_pages;
    if (s.end == kr.sink && hi > kr.sink && s.n < most) {
      const int32_t end = int32_t(min(int64_t(last) + 1, int64_t(s.p0 + most - s.n) << shift));
      s.end = kr.sink + (end - kr.lo);
      s.n += ((end - 1) >> shift) - s.p0 + 1;
    }
    return s;
  }
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

// The larger of the values of lanes 16 apart, in both.
__device__ inline float max_of_16s(float x) {
  const uint32_t b = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
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
__device__ inline float log_sum(float top, float sum, float c2, float lift) {
  return sum == 0.f ? -INFINITY : (top * c2 + (__log2f(sum) - lift)) * kLn2;
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
  if (c == 0 && a.lse) a.lse[t * a.n_heads + h] = log_sum(top, sum, a.c2, a.lift);
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
  const int32_t len = kr.length();
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
  const int32_t len = kr.length();
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

// What a plan goes by beside the step.
struct Shape {
  int32_t n_heads, n_kv_heads, head_dim, window, sinks;
  int32_t few_most;   // keys of a split of few rows, at most
  int32_t few_whole;  // keys times head_dim that eight waves take without a split
  int32_t few_once;     // keys that are not split where the card is full without, at most
  int32_t chunk_want;   // work-groups wanted of several requests' chunks
  int32_t chunk_least;  // keys of a split of chunks, at least
};
Shape shape_of(const fs_step *s, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
               int32_t window, int32_t sinks, int32_t few_most, int32_t few_whole,
               int32_t few_once, int32_t chunk_want, int32_t chunk_least) {
  window = limited(window, s);
  sinks = window == 0 ? 0 : sinks < s->max_kv ? sinks : s->max_kv;
  return {n_heads, n_kv_heads, head_dim, window, sinks, few_most, few_whole, few_once, chunk_want,
          chunk_least};
}

Plan plan(const fs_step *s, const Shape &c) {
  Plan p = {};
  const int32_t G = c.n_heads / c.n_kv_heads;
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
    const int64_t k = c.window ? int64_t(c.window) + c.sinks + tokens : s->max_kv;
    return int32_t(k < s->max_kv ? k : s->max_kv);
  };
  auto split_of = [&](int64_t blocks, int32_t len, int32_t want, int32_t least, int32_t most,
                      int64_t rows, int32_t &split, int32_t &splits) {
    const int64_t bytes = rows * c.n_heads * (c.head_dim + 2) * 4;  // of one split
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
    const int64_t blocks = int64_t(p.few_seqs) * c.n_kv_heads;
    const int32_t len = keys(p.few_tokens);
    split_of(blocks, len, 1024, 512, c.few_most, int64_t(s->n_seqs) * p.few_tokens, p.few_split,
             p.few_splits);
    // Not split where every compute unit has a work-group without, and the longest few enough
    // keys for them: no join.  (4 bits: 64 requests of up to 16,384 tokens, 8 heads of 128, a
    // window of 700 14.2 us, 16.2 in two splits, of 1,500 19.1 and 21.6; 40 of 1,500, 16 heads,
    // 33 and 40; 64 of 2,000 34.6 and 39.3, but 33 of 2,000 27.2 and 24.6.  16 bits with sinks:
    // a window of 1,000 30.2 and 33.4, and of 1,500 over 264 work-groups 29.3 and 25.2.)
    const int64_t once = 1024 + 2 * blocks;
    if (blocks > 256 && p.few_splits > 1 && len <= (once < c.few_once ? once : c.few_once)) {
      p.few_split = c.few_once;
      p.few_splits = 1;
    }
    // Up to 1,024 keys (2,048 of head_dim 64) with a compute unit for each work-group: eight
    // waves and no join.  (4 requests, 8 heads of 128: 500 keys 8.9 us, 9.8 with four waves;
    // 1,000 keys 11.5 and, in two splits, 13.5; 30 requests of 1,000 13.4 and 17.1; 1,500 keys
    // whole 14.5, in splits 13.8.  Of 64: 1,400 keys 10.3 and 13.2, 2,000 12.9 and 14.1.)
    const int32_t whole = c.few_whole / c.head_dim;
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
    p.chunk_rows = c.head_dim == 128 && p.few_seqs == 0 &&
                           int64_t(tiles(256)) * c.n_kv_heads >= 256
                       ? 256
                       : 128;
    p.chunk_tiles = tiles(p.chunk_rows);
    // 512 work-groups wanted, of at least 1,024 keys over the 16-bit cache (300 rows over 20,000
    // keys: 134 us, 154 with 256 work-groups, 144 with 1,024)
    const int32_t toks = p.chunk_rows / G + 2;
    split_of(int64_t(p.chunk_tiles) * c.n_kv_heads, keys(most < toks ? most : toks),
             p.chunk_seqs > 1 ? c.chunk_want : 512, c.chunk_least, 1 << 30,
             s->q_off_h[s->n_seqs], p.chunk_split, p.chunk_splits);
  }
  return p;
}

size_t round256(size_t x) { return (x + 255) / 256 * 256; }

// Bytes of the partial results: [rows][D] and [rows][2] floats of each kind.
struct Space {
  size_t few_o, few_ml, chunk_o, chunk_ml;
  size_t total() const { return few_o + few_ml + chunk_o + chunk_ml; }
};
Space space(const Plan &p, const fs_step *s, const Shape &c) {
  Space w = {};
  if (p.few_splits > 1) {
    const size_t r = size_t(p.few_splits) * s->n_seqs * p.few_tokens * c.n_heads;
    w.few_o = round256(r * c.head_dim * 4);
    w.few_ml = round256(r * 8);
  }
  if (p.chunk_splits > 1) {
    const size_t r = size_t(p.chunk_splits) * s->q_off_h[s->n_seqs] * c.n_heads;
    w.chunk_o = round256(r * c.head_dim * 4);
    w.chunk_ml = round256(r * 8);
  }
  return w;
}
// The arguments that do not depend on the kind of cache.
void fill_args(AttnArgs &a, const Plan &p, const Space &w, const Shape &c, const fs_step *s,
               float scale, const void *q, int64_t q_stride, void *out, int64_t out_stride,
               float *lse, void *ws, int32_t *err) {
  a.q_off = s->q_off;
  a.kv_len = s->kv_len;
  a.n_seqs = s->n_seqs;
  a.max_kv = s->max_kv;
  a.rows = s->q_off_h[s->n_seqs];
  a.n_heads = c.n_heads;
  a.window = c.window;
  a.sinks = c.sinks;
  a.group = c.n_heads / c.n_kv_heads;
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
}

}  // namespace

}  // namespace fs
