// A projection with every request's own low-rank adapter beside the shared weight:
//   y = x W^T + scale_a (x A_a^T) B_a^T,   a = the row's request's adapter.
// Two launches.  k_shrink makes h = scale x A_a^T per request in fp32 and stores it as the
// sum of two 16-bit values (in half precision in units of a power of two of the row's own),
// with the row's adapter and rank beside it.  The product then runs over K and goes on over
// the few columns of h against B_a, so y is written once and never read:
//   k_shrink       16 rows of one request a work-group; its waves share out K and join in
//                  LDS.  Bound by the bytes of x where there are many rows (16,384 rows of
//                  4,096: 134 MB in 38 us, 3.6 TB/s), by one tile's chain where there are few
//                  (5.6 us).
//   k_linear_few   up to 64 rows: bound by the bytes of W, and at a few MB by what a
//                  work-group can have under way (64 rows, 4,096 x 6,144: 50 MB in 17 to 20
//                  us).  A work-group takes 16 to 64 columns of y; its four waves share out K
//                  and join in LDS.
//   k_linear_tile  more rows: bound by the matrix cores and LDS together.  W and x go through
//                  LDS in tiles (16,384 x 4,096 x 4,096: 467 us and the shrink's 37, 487 to
//                  510 a call from card to card, 1.1 PFLOP/s, the matrix cores busy for 63 %
//                  of the cycles; its loads alone take 404 us, its products alone 419).  Eight
//                  waves with tiles of 128 x 64 each read LDS least for a product.
// W is the first operand (its rows are y's columns), so a lane holds neighbouring columns
// of one row of y.
#include "fs_engine.h"

namespace fs {

namespace {

struct LinArgs {
  const int32_t *q_off, *adapter, *rank;
  const float *scale;
  int32_t n_seqs, rows, K, N, n_adapters, R;  // R: max_rank (0: no adapters)
  const short *x, *w, *a, *b;
  short *y;
  short *h;         // [rows][2R]: high parts, low parts
  // [rows up to a multiple of 16]: the row's adapter (-1: none); its rank, and from bit 8 on
  // the exponent of what h counts in (half precision; 1 in bfloat16)
  int2 *row_ad;
  int64_t x_stride, y_stride;
  int32_t *err;
};

// Adapter of a request and its rank; -1 when it has none (a bad id raises *code).
__device__ inline int32_t adapter_of(const LinArgs &g, int32_t s, int32_t &rank, int32_t &code) {
  rank = 0;
  if (g.n_adapters == 0) return -1;
  const int32_t a = __ldg(g.adapter + s);
  if (a < 0 || a >= g.n_adapters) {
    if (a != -1) code = FS_E_RANGE;
    return -1;
  }
  rank = g.rank ? __ldg(g.rank + a) : g.R;
  if (rank < 0 || rank > g.R) {
    code = FS_E_RANGE;
    rank = 0;
  }
  return a;
}

// Which 16-byte chunk of its row lies in place c of row r of an LDS tile (and the other way
// round): 16 rows' chunks of one column fall on different banks.
template <int BK>
__device__ inline int place_of(int r, int c) {
  return BK == 64 ? c ^ ((r >> 1) & 7) : c ^ ((r >> 2) & 3);
}

// acc[m][n] += W x^T over this wave's share of K: MT tiles of 16 rows of x, NT of 16 rows of
// w.  The waves take 64 of K in turn, each through STAGES buffers of its own that are filled
// STAGES - 1 steps ahead, so they never wait for each other.  (Straight from memory in the
// matrix cores' layout, 16 lanes would touch 16 rows: a quarter of the cache's rate.)
// `meanwhile` runs once the first loads are under way.
template <bool BF, int MT, int NT, int WAVES, int STAGES, class F>
__device__ void share_of_k(const short *x, int64_t x_stride, int x_rows, const short *w, int w_rows,
                           int K, int wave, short *lds, f32x4 (&acc)[MT][NT], F meanwhile) {
  constexpr int TILE = 16 * 64, STEP = (MT + NT) * TILE, LOADS = 2 * (MT + NT);
  const int lane = threadIdx.x & 63, r16 = lane & 15, g4 = lane >> 4;
  short *mine = lds + wave * (STAGES * STEP);
  const uint32_t at = lds_address(mine);
  uint32_t off[LOADS];
  int col[2];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int r = i * 8 + (lane >> 3);  // of x's tiles, then w's
    col[i & 1] = place_of<64>(r & 15, lane & 7) * 8;
    off[i] = i < 2 * MT ? uint32_t(min(r, x_rows - 1) * x_stride + col[i & 1]) * 2
                        : uint32_t(min(r - MT * 16, w_rows - 1) * K + col[i & 1]) * 2;
  }
  const int slices = (K + 63) / 64, n = slices > wave ? (slices - wave + WAVES - 1) / WAVES : 0;
  auto issue = [&](int t) {
    const int k = (wave + t * WAVES) * 64;
    const uint32_t to = at + (t % STAGES) * STEP * 2;
    if (k + 64 <= K) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) load_to_lds((i < 2 * MT ? x : w) + k, off[i], to + i * 1024);
    } else {  // past the end of K: the last chunk of the row, its products are masked
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
        load_to_lds((i < 2 * MT ? x : w) + k, off[i] + 2 * min(0, K - 8 - k - col[i & 1]),
                    to + i * 1024);
    }
  };
  auto multiply = [&](int t, bool whole) {
    const short *b = mine + (t % STAGES) * STEP;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int c = u * 4 + g4, place = r16 * 64 + place_of<64>(r16, c) * 8;
      s16x8 xf[MT], wf[NT];
#pragma unroll
      for (int m = 0; m < MT; ++m) xf[m] = *reinterpret_cast<const s16x8 *>(b + m * TILE + place);
#pragma unroll
      for (int j = 0; j < NT; ++j)
        wf[j] = *reinterpret_cast<const s16x8 *>(b + (MT + j) * TILE + place);
      if (!whole) {
        const s16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
        const bool in = (wave + t * WAVES) * 64 + c * 8 < K;
#pragma unroll
        for (int m = 0; m < MT; ++m) xf[m] = in ? xf[m] : zero;
#pragma unroll
        for (int j = 0; j < NT; ++j) wf[j] = in ? wf[j] : zero;
      }
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[m][j] = mfma_16x16x32<BF>(wf[j], xf[m], acc[m][j]);
    }
  };
#pragma unroll
  for (int t = 0; t < STAGES - 1; ++t)
    if (t < n) issue(t);
  meanwhile();
  int t = 0;
  for (; t + STAGES - 1 < n; ++t) {
    reads_done();
    issue(t + STAGES - 1);
    wait_own<(STAGES - 1) * LOADS>();
    multiply(t, true);
  }
  wait_own<0>();
  for (; t < n; ++t) {
    multiply(t, (wave + t * WAVES + 1) * 64 <= K);
  }
}

// One request's rows, 16 at a time, against its adapter's A; the waves share out K and join
// in LDS.  JT: 16-column tiles of h.
template <bool BF, int JT, int WAVES, int STAGES>
__global__ void __launch_bounds__(WAVES * 64) k_shrink(LinArgs g) {
  constexpr int LOADED = WAVES * STAGES * (1 + JT) * 16 * 64;
  __shared__ __align__(16) short lds[LOADED];
  static_assert(LOADED >= WAVES * JT * 256 * 2 + 32, "room for the partial sums and `most`");
  uint32_t *most = reinterpret_cast<uint32_t *>(lds + LOADED) - 16;  // rows' largest, as bits
  const RowTile t = row_tile<4>(g.q_off, g.n_seqs, blockIdx.x);
  if (t.rows <= 0) return;
  int32_t code = 0, rank;
  const int32_t ad = adapter_of(g, t.s, rank, code);
  if (threadIdx.x == 0) raise_err(g.err, code);
  if (ad < 0 || rank == 0) {  // h of such rows is not looked at
    if (threadIdx.x < t.rows) g.row_ad[t.row0 + threadIdx.x] = {-1, 0};
    return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  f32x4 acc[1][JT] = {};
  share_of_k<BF, 1, JT, WAVES, STAGES>(g.x + int64_t(t.row0) * g.x_stride, g.x_stride, t.rows,
                                       g.a + int64_t(ad) * g.R * g.K, rank, g.K, wave, lds, acc,
                                       [] {});
  __syncthreads();
  f32x4 *part = reinterpret_cast<f32x4 *>(lds);
#pragma unroll
  for (int j = 0; j < JT; ++j) part[(wave * JT + j) * 64 + lane] = acc[0][j];
  if (threadIdx.x < 16) most[threadIdx.x] = 0;
  __syncthreads();
  const float scale = g.scale ? __ldg(g.scale + ad) : 1.f;
  constexpr int PER = (JT + WAVES - 1) / WAVES;
  f32x4 v[PER];
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int e = threadIdx.x + p * WAVES * 64, row = e & 15, j0 = (e >> 4) * 4;
    if (e >= JT * 64) continue;
    v[p] = part[e];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v[p] += part[w * JT * 64 + e];
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[p][i] = j0 + i < rank ? v[p][i] * scale : 0.f;
      m = fmaxf(m, fabsf(v[p][i]));
    }
    if (!BF) atomicMax(&most[row], __float_as_uint(m));
  }
  if (!BF) __syncthreads();
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int e = threadIdx.x + p * WAVES * 64, row = e & 15, j0 = (e >> 4) * 4;
    if (e >= JT * 64 || row >= t.rows || j0 >= g.R) continue;
    // half precision: a power of two brings the row's largest to between 2^14 and 2^15, so
    // that none is beyond the range and the low parts are not below it
    // (a unit of at least 2^-40: sums are divided by it)
    const uint32_t top = BF ? 0 : most[row] >> 23, ex = top < 101 ? 101 : top;
    const float up = BF || ex == 255 ? 1.f : __uint_as_float((268 - ex) << 23);
    const uint32_t unit = BF || ex == 255 ? 127 : ex - 14;
    s16x4 hi, lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float f = v[p][i] * up;
      hi[i] = to_16<BF>(f);
      const float left = f - to_f32<BF>(hi[i]);
      lo[i] = to_16<BF>(fabsf(left) < INFINITY ? left : 0.f);  // an infinite h has no low part
    }
    short *hp = g.h + int64_t(t.row0 + row) * (2 * g.R) + j0;
    *reinterpret_cast<s16x4 *>(hp) = hi;
    *reinterpret_cast<s16x4 *>(hp + g.R) = lo;
    if (j0 == 0) g.row_ad[t.row0 + row] = {ad, int32_t(rank | unit << 8)};
  }
}

__device__ inline int32_t rank_in(int32_t packed) { return packed & 255; }
__device__ inline float unit_in(int32_t packed) { return __uint_as_float(packed >> 8 << 23); }

// B_a[n][j .. j + 7] (another place's at j = R), and 0 for its columns at and beyond the rank.
__device__ inline s16x8 load_b(const LinArgs &g, int32_t ad, int32_t n, int j) {
  return *reinterpret_cast<const s16x8 *>(g.b + (int64_t(ad) * g.N + n) * g.R + min(j, g.R - 8));
}
__device__ inline s16x8 within_rank(s16x8 v, int j, int32_t rank) {
  if (j + 8 > rank)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = j + i < rank ? v[i] : short(0);
  return v;
}
// ---- few rows: all of them, in MT tiles of 16, by NT tiles of 16 columns, four waves
template <bool BF, int MT, int NT, int STAGES>
__global__ void __launch_bounds__(256) k_linear_few(LinArgs g) {
  __shared__ __align__(16) short lds[4 * STAGES * (MT + NT) * 16 * 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g4 = lane >> 4;
  const int n0 = blockIdx.x * (NT * 16);
  const s16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
  // the adapters of the tile of rows that this wave deals with
  const int my = wave % MT, my_row = my * 16 + r;
  const int2 ad = g.n_adapters > 0 && my_row < g.rows ? g.row_ad[my_row] : int2{-1, 0};
  f32x4 acc[MT][NT] = {};
  // The distinct adapters of a tile's rows, shared out over the 4 / MT waves that hold the
  // tile, while the first loads for the product over K are under way.  Every row is multiplied
  // with each of them and takes only its own one's result (a product of 0 with another
  // adapter's infinity would be NaN).  Four adapters' loads go side by side, for WIDE times 4
  // chunks of 8 columns (R/8 high ones, then R/8 low ones): 3 us of 20 at 64 rows of 8
  // adapters of rank 16, 9 at rank 64.
  auto adapters = [&] {
    uint64_t left = __ballot(ad.x >= 0);
    if (left) {
      constexpr int WIDE = NT == 1 ? 2 : 1;
      const int chunks = g.R / 8;
      const short *hp = g.h + int64_t(min(my_row, g.rows - 1)) * (2 * g.R);
      f32x4 sum[NT] = {};
      for (int turn = 0; left;) {
        int32_t who[4] = {-1, -1, -1, -1}, rank[4] = {0, 0, 0, 0};
        int found = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          while (left) {
            const int first = __builtin_ctzll(left);
            const int32_t a = __builtin_amdgcn_readlane(ad.x, first);
            left &= ~__ballot(ad.x == a);
            if (turn++ % (4 / MT) == wave / MT) {
              who[i] = a;
              rank[i] = rank_in(__builtin_amdgcn_readlane(ad.y, first));
              ++found;
              break;
            }
          }
        }
        if (found == 0) break;
        const short *bp[4][NT];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const int col = min(n0 + n * 16 + r, g.N - 1);
            bp[i][n] = g.b + (int64_t(max(who[i], 0)) * g.N + col) * g.R;
          }
        f32x4 one[4][NT] = {};
        for (int c0 = g4; c0 < (2 * chunks + 3) / 4 * 4; c0 += 4 * WIDE) {
          s16x8 hv[WIDE], bv[WIDE][4][NT];
          int j[WIDE];
#pragma unroll
          for (int u = 0; u < WIDE; ++u) {
            const int c = c0 + u * 4;
            const bool in = c < 2 * chunks;
            j[u] = in ? (c < chunks ? c : c - chunks) * 8 : g.R;
            hv[u] = *reinterpret_cast<const s16x8 *>(hp + (in ? c : 0) * 8);
            hv[u] = in ? hv[u] : zero;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int n = 0; n < NT; ++n)
                bv[u][i][n] = *reinterpret_cast<const s16x8 *>(bp[i][n] + min(j[u], g.R - 8));
          }
#pragma unroll
          for (int u = 0; u < WIDE; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int n = 0; n < NT; ++n)
                one[i][n] =
                    mfma_16x16x32<BF>(within_rank(bv[u][i][n], j[u], rank[i]), hv[u], one[i][n]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int n = 0; n < NT; ++n)
            if (ad.x >= 0 && ad.x == who[i]) sum[n] += one[i][n];
      }
      const float unit = !BF && ad.x >= 0 ? unit_in(ad.y) : 1.f;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
          if (m == my) acc[m][n] += sum[n] * unit;
    }
  };
  share_of_k<BF, MT, NT, 4, STAGES>(g.x, g.x_stride, g.rows, g.w + int64_t(n0) * g.K, g.N - n0,
                                    g.K, wave, lds, acc, adapters);
  __syncthreads();
  f32x4 *part = reinterpret_cast<f32x4 *>(lds);
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) part[(wave * MT * NT + m * NT + n) * 64 + lane] = acc[m][n];
  __syncthreads();
  for (int t = wave; t < MT * NT; t += 4) {
    f32x4 v = part[t * 64 + lane];
#pragma unroll
    for (int w = 1; w < 4; ++w) v += part[(w * MT * NT + t) * 64 + lane];
    const int row = (t / NT) * 16 + r, n = n0 + (t % NT) * 16 + (lane >> 4) * 4;
    if (row < g.rows && n < g.N) {
      s16x4 o;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = to_16<BF>(v[i]);
      *reinterpret_cast<s16x4 *>(g.y + int64_t(row) * g.y_stride + n) = o;
    }
  }
}

// The distinct adapters of a wave's 32 rows in steps of two chunks of 8 columns (R/8 chunks of
// h's high parts, then R/8 of its low ones).
struct Steps {
  int2 ad;        // the lane's row's adapter and rank
  uint64_t left;  // lanes whose adapter is still to come
  int each, at;   // an adapter's steps, the next one
  int32_t who = -1, rank = 0;
  __device__ Steps(const LinArgs &g, int2 row_ad) : ad(row_ad) {
    left = __ballot(ad.x >= 0);
    each = at = g.R / 8;
  }
  __device__ bool done() const { return at == each && !left; }
  // The next step's adapter (-1, at step 0: none is left), its step and its rank.
  __device__ int32_t next(int &step, int32_t &its_rank) {
    if (at == each) {
      who = -1;
      if (left) {
        const int first = __builtin_ctzll(left);
        who = __builtin_amdgcn_readlane(ad.x, first);
        rank = rank_in(__builtin_amdgcn_readlane(ad.y, first));
        left &= ~__ballot(ad.x == who);
        at = 0;
      }
    }
    step = who < 0 ? 0 : at;
    its_rank = rank;
    at += who >= 0;
    return who;
  }
};

// ---- many rows: BM rows by BN columns a work-group, K in steps of BK through STAGES LDS
// buffers that are filled STAGES - 1 steps ahead; a wave takes WM rows by WN columns.
template <bool BF, int BM, int BN, int WM, int WN, int BK, int STAGES>
__global__ void __launch_bounds__((BM / WM) * (BN / WN) * 64, 2) k_linear_tile(LinArgs g) {
  constexpr int WAVES = (BM / WM) * (BN / WN);
  constexpr int MT = WM / 32, NT = WN / 32;
  constexpr int CH = BK / 8, RW = 64 / CH;  // chunks of a row, rows of a wave's load
  constexpr int LX = BM / RW / WAVES, LW = BN / RW / WAVES;  // a wave's loads of a step
  __shared__ __align__(16) short xs[STAGES][BM * BK], ws[STAGES][BN * BK];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r32 = lane & 31, h2 = lane >> 5;

  // Work-groups go to the 8 dies in turn: each die takes a run of neighbouring tiles, in
  // strips of 8 row tiles, so that its L2 serves the x and W they share.
  const int tm = (g.rows + BM - 1) / BM, tn = (g.N + BN - 1) / BN, total = tm * tn;
  int id = blockIdx.x;
  {
    const int die = id & 7, per = total >> 3, extra = total & 7;
    id = die * per + min(die, extra) + (id >> 3);
  }
  const int strip = 8 * tn, first = id / strip * 8, width = min(8, tm - first);
  const int m0 = (first + (id % strip) % width) * BM, n0 = (id % strip) / width * BN;

  const int wm = (wave % (BM / WM)) * WM, wn = (wave / (BM / WM)) * WN;
  f32x16 acc[MT][NT] = {};
  // this lane's row and chunk of each of the wave's loads, as bytes from the tile's start
  uint32_t xo[LX], wo[LW];
  int xc[LX], wc[LW];
#pragma unroll
  for (int i = 0; i < LX; ++i) {
    const int r = (wave * LX + i) * RW + lane / CH;
    xc[i] = place_of<BK>(r, lane % CH) * 8;
    xo[i] = uint32_t((min(m0 + r, g.rows - 1) - m0) * g.x_stride + xc[i]) * 2;
  }
#pragma unroll
  for (int i = 0; i < LW; ++i) {
    const int r = (wave * LW + i) * RW + lane / CH;
    wc[i] = place_of<BK>(r, lane % CH) * 8;
    wo[i] = uint32_t((min(n0 + r, g.N - 1) - n0) * g.K + wc[i]) * 2;
  }
  int2 ad[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int row = m0 + wm + m * 32 + r32;
    ad[m] = g.n_adapters > 0 && row < g.rows ? g.row_ad[row] : int2{-1, 0};
  }
  const short *x0 = g.x + int64_t(m0) * g.x_stride, *w0 = g.w + int64_t(n0) * g.K;
  const uint32_t xs_at = lds_address(&xs[0][wave * LX * RW * BK]),
                 ws_at = lds_address(&ws[0][wave * LW * RW * BK]);
  auto issue = [&](int step) {
    const int k = step * BK, s = step % STAGES;
    if (k + BK <= g.K) {
#pragma unroll
      for (int i = 0; i < LX; ++i)
        load_to_lds(x0 + k, xo[i], xs_at + (s * BM + i * RW) * BK * 2);
#pragma unroll
      for (int i = 0; i < LW; ++i)
        load_to_lds(w0 + k, wo[i], ws_at + (s * BN + i * RW) * BK * 2);
    } else {  // past the end of K: the last chunk of the row, its products are masked
#pragma unroll
      for (int i = 0; i < LX; ++i)
        load_to_lds(x0 + k, xo[i] + 2 * min(0, g.K - 8 - k - xc[i]),
                    xs_at + (s * BM + i * RW) * BK * 2);
#pragma unroll
      for (int i = 0; i < LW; ++i)
        load_to_lds(w0 + k, wo[i] + 2 * min(0, g.K - 8 - k - wc[i]),
                    ws_at + (s * BN + i * RW) * BK * 2);
    }
  };
  auto multiply = [&](int step, bool whole, auto meanwhile) {
    const short *xt = xs[step % STAGES], *wt = ws[step % STAGES];
    constexpr int AHEAD = MT * NT == 1 ? BK / 16 : 2;
    s16x8 xf[AHEAD][MT], wf[AHEAD][NT];
    auto operands = [&](int u) {
      const int c = u * 2 + h2;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int r = wn + n * 32 + r32;
        wf[u % AHEAD][n] = *reinterpret_cast<const s16x8 *>(wt + r * BK + place_of<BK>(r, c) * 8);
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int r = wm + m * 32 + r32;
        xf[u % AHEAD][m] = *reinterpret_cast<const s16x8 *>(xt + r * BK + place_of<BK>(r, c) * 8);
      }
      if (!whole) {
        const s16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
        const bool in = step * BK + c * 8 < g.K;
#pragma unroll
        for (int m = 0; m < MT; ++m) xf[u % AHEAD][m] = in ? xf[u % AHEAD][m] : zero;
#pragma unroll
        for (int n = 0; n < NT; ++n) wf[u % AHEAD][n] = in ? wf[u % AHEAD][n] : zero;
      }
    };
    // The next 16 columns' operands are read while these are multiplied; a small tile's all
    // at once.  The loads of a later step are issued while the first are read (before them:
    // 100 rows of 4,096 by 6,144 columns 28.1 us, so 27.1; 16,384 by 4,096 515 and 505).
#pragma unroll
    for (int u = 0; u < AHEAD - 1; ++u) operands(u);
    if (AHEAD == BK / 16) operands(AHEAD - 1);
    meanwhile();
#pragma unroll
    for (int u = 0; u < BK / 16; ++u) {
      if (AHEAD < BK / 16 && u + AHEAD - 1 < BK / 16) operands(u + AHEAD - 1);
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
          acc[m][n] = mfma_32x32x16<BF>(wf[u % AHEAD][n], xf[u % AHEAD][m], acc[m][n]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  const int steps = (g.K + BK - 1) / BK, full = g.K / BK;
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s)
    if (s < steps) issue(s);
  int step = 0;
  for (; step + STAGES - 1 < steps; ++step) {
    wait_loads<(STAGES - 2) * (LX + LW)>();
    multiply(step, true, [&] { issue(step + STAGES - 1); });
  }
  for (; step < steps; ++step) {
    wait_loads<0>();
    multiply(step, step < full, [] {});
  }
  const int chunks = g.R / 8;
  constexpr int UNITS = MT * NT == 1 ? 4 : 2;  // steps whose loads go side by side
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int row = m0 + wm + m * 32 + r32;
    const short *hp = g.h + int64_t(min(row, g.rows - 1)) * (2 * g.R);
    Steps adapters(g, ad[m]);
    if (!adapters.left) continue;
    const float unit = !BF && ad[m].x >= 0 ? unit_in(ad[m].y) : 1.f;
    int32_t who[UNITS], rank[UNITS];
    int at[UNITS], j[UNITS];
    s16x8 hv[UNITS], bv[UNITS][NT];
    auto fetch = [&] {
#pragma unroll
      for (int i = 0; i < UNITS; ++i) who[i] = adapters.next(at[i], rank[i]);
#pragma unroll
      for (int i = 0; i < UNITS; ++i) {
        const int c = at[i] * 2 + h2;
        hv[i] = *reinterpret_cast<const s16x8 *>(hp + c * 8);
        j[i] = (c < chunks ? c : c - chunks) * 8;
#pragma unroll
        for (int n = 0; n < NT; ++n)
          bv[i][n] = load_b(g, max(who[i], 0), min(n0 + wn + n * 32 + r32, g.N - 1), j[i]);
      }
    };
    const int32_t first = __builtin_amdgcn_readlane(ad[m].x, __builtin_ctzll(adapters.left));
    if (__all(ad[m].x == first || row >= g.rows)) {  // all in one sum
      if (!BF)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[m][n] *= 1.f / unit;
      while (!adapters.done()) {
        fetch();
#pragma unroll
        for (int i = 0; i < UNITS; ++i)
          if (who[i] >= 0)
#pragma unroll
            for (int n = 0; n < NT; ++n)
              acc[m][n] =
                  mfma_32x32x16<BF>(within_rank(bv[i][n], j[i], rank[i]), hv[i], acc[m][n]);
      }
      if (!BF)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[m][n] *= unit;
      continue;
    }
    // every row with each adapter; it takes only its own one's result
    f32x16 one[NT] = {};
    while (!adapters.done()) {
      fetch();
#pragma unroll
      for (int i = 0; i < UNITS; ++i) {
        if (who[i] < 0) continue;
#pragma unroll
        for (int n = 0; n < NT; ++n)
          one[n] = mfma_32x32x16<BF>(within_rank(bv[i][n], j[i], rank[i]), hv[i], one[n]);
        if (at[i] + 1 < adapters.each) continue;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          if (ad[m].x == who[i]) acc[m][n] += one[n] * unit;
          one[n] = f32x16{};
        }
      }
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int row = m0 + wm + m * 32 + r32;
    if (row >= g.rows) continue;
    short *yp = g.y + int64_t(row) * g.y_stride;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int col = n0 + wn + n * 32 + i * 8 + h2 * 4;
        s16x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = to_16<BF>(acc[m][n][i * 4 + e]);
        if (col < g.N) *reinterpret_cast<s16x4 *>(yp + col) = o;
      }
  }
}

template <bool BF, int JT>
void shrink(const LinArgs &g, const fs_step *st, hipStream_t stream) {
  const int64_t tiles = row_tiles(st, 4);
  // few tiles: more waves share out K, so that one tile's time is short (as LDS allows);
  // many: the loads of several steps are under way.  (The two lie within 1 % of the whole
  // call on either side: 137 tiles 40.9 against 41.3 us, 512 259.5 against 262.)
  constexpr int kMost = JT == 1 ? 16 : JT <= 4 ? 8 : 4;
  constexpr int kStages = JT == 1 ? 4 : JT == 2 ? 3 : 2;
  if (tiles <= 512)
    hipLaunchKernelGGL((k_shrink<BF, JT, kMost, 2>), dim3(tiles), dim3(kMost * 64), 0, stream, g);
  else
    hipLaunchKernelGGL((k_shrink<BF, JT, 4, kStages>), dim3(tiles), dim3(256), 0, stream, g);
}

// Columns of a work-group: each reads all of x, so few rows take the least columns, and more
// take 16 while two of them on each compute unit hold all columns, else 48 or 64, one on each
// compute unit, as fewer rounds of its time ask (with the shrink, K = 4,096, 64 rows:
//   columns        6,144   9,000  14,336  20,000  28,672
//   16 at a time    24.6    37.5    55.7    69.5    95.5 us
//   32              25.0    48.0    54.1    79.4   105.1
//   48              24.8    30.0    58.1    64.6    91.0
//   64              27.6    33.6    41.8    76.1    81.9
// 16 rows by 28,672: 58 us with 16 columns, 70 with 32, 57 with 64; 64 rows on their tiles of
// k_linear_tile: 29.9 us for 6,144 columns, 39.0 for 14,336, 85.5 for 28,672).
template <bool BF, int MT>
void few(const LinArgs &g, hipStream_t stream) {
  constexpr int kStages = MT == 4 ? 2 : MT == 2 ? 3 : 4;  // 64 to 80 KB of LDS for 16 columns
  auto groups = [&](int cols) { return dim3((g.N + cols - 1) / cols); };
  if (MT == 1 || g.N <= 512 * 16)
    hipLaunchKernelGGL((k_linear_few<BF, MT, 1, kStages>), groups(16), dim3(256), 0, stream, g);
  else if constexpr (MT > 1) {
    const int cus = 256, by48 = (g.N + cus * 48 - 1) / (cus * 48),
              by64 = (g.N + cus * 64 - 1) / (cus * 64);
    if (by48 * 3 <= by64 * 4)
      hipLaunchKernelGGL((k_linear_few<BF, MT, 3, 2>), groups(48), dim3(256), 0, stream, g);
    else
      hipLaunchKernelGGL((k_linear_few<BF, MT, 4, 2>), groups(64), dim3(256), 0, stream, g);
  }
}

template <bool BF>
void run(const LinArgs &g, const fs_step *st, hipStream_t stream) {
  if (g.n_adapters > 0) {
    if (g.R <= 16)
      shrink<BF, 1>(g, st, stream);
    else if (g.R <= 32)
      shrink<BF, 2>(g, st, stream);
    else if (g.R <= 64)
      shrink<BF, 4>(g, st, stream);
    else
      shrink<BF, 8>(g, st, stream);
  }
  if (g.rows <= 64) {
    if (g.rows <= 16)
      few<BF, 1>(g, stream);
    else if (g.rows <= 32)
      few<BF, 2>(g, stream);
    else
      few<BF, 4>(g, stream);
    return;
  }
  // The largest tiles that still occupy three quarters of the compute units (K = 4,096: 1,024
  // tiles of 256 take 516 us, of 128 587 and of 64 902; 2,048 rows by 4,096 columns, 128 tiles
  // of 256, 106, 75 and 114 us; K = 2,048, 500 rows by 2,560 columns: - , 34.0 and 22.7,
  // and 1,000 rows 34.7 with 64 and 32.2 with 128 by 96).
  auto tiles = [&](int64_t t) { return ((g.rows + t - 1) / t) * ((g.N + t - 1) / t); };
  const int64_t narrow = (g.rows + 127) / 128 * int64_t((g.N + 95) / 96);  // of 128 by 96
  if (tiles(256) >= 192)
    hipLaunchKernelGGL((k_linear_tile<BF, 256, 256, 128, 64, 64, 2>), dim3(tiles(256)), dim3(512),
                       0, stream, g);
  else if (narrow >= 192) {
    // 96 columns for 128 where that takes no more rounds of two work-groups a compute unit, or
    // few enough (a round of them takes 0.9 of the time of one of the others: K = 2,048, 1,999
    // rows by 2,560 columns 39.7 and 42.3 us; K = N = 4,096: 1,500 rows 98 and 68.5, 2,500 107
    // and 115.5)
    if ((narrow + 511) / 512 * 115 < (tiles(128) + 511) / 512 * 128)
      hipLaunchKernelGGL((k_linear_tile<BF, 128, 96, 32, 96, 64, 2>), dim3(narrow), dim3(256), 0,
                         stream, g);
    else
      hipLaunchKernelGGL((k_linear_tile<BF, 128, 128, 64, 64, 64, 2>), dim3(tiles(128)), dim3(256),
                         0, stream, g);
  } else
    hipLaunchKernelGGL((k_linear_tile<BF, 64, 64, 32, 32, 64, 4>), dim3(tiles(64)), dim3(256), 0,
                       stream, g);
}

}  // namespace

size_t adapter_workspace_bytes(const fs_step *s, const fs_adapters *ad) {
  if (ad->n_adapters == 0) return 0;
  const size_t rows = s->q_off_h[s->n_seqs], whole = (rows + 15) / 16 * 16;
  return rows * ad->max_rank * 4 + whole * 8;
}

hipError_t launch_adapter_linear(const fs_step *s, const fs_adapters *ad, const void *x,
                                 int64_t x_stride, const void *w, void *y, int64_t y_stride,
                                 void *ws, int32_t *err, hipStream_t stream) {
  LinArgs g;
  g.q_off = s->q_off;
  g.adapter = ad->adapter;
  g.rank = ad->rank;
  g.scale = ad->scale;
  g.n_seqs = s->n_seqs;
  g.rows = s->q_off_h[s->n_seqs];
  g.K = ad->in_features;
  g.N = ad->out_features;
  g.n_adapters = ad->n_adapters;
  g.R = ad->n_adapters > 0 ? ad->max_rank : 0;
  g.x = static_cast<const short *>(x);
  g.w = static_cast<const short *>(w);
  g.a = static_cast<const short *>(ad->a);
  g.b = static_cast<const short *>(ad->b);
  g.y = static_cast<short *>(y);
  g.h = static_cast<short *>(ws);
  g.row_ad = reinterpret_cast<int2 *>(g.h + size_t(g.rows) * g.R * 2);
  g.x_stride = x_stride;
  g.y_stride = y_stride;
  g.err = err;
  if (ad->dtype == FS_BF16)
    run<true>(g, s, stream);
  else
    run<false>(g, s, stream);
  return hipGetLastError();
}

}  // namespace fs
