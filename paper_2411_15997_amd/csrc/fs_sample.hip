// The next token of each row from its logits and one given random number, in whole-number
// weights (2^40 for the largest logit): every sum is exact, so the kept set and the token
// do not depend on the order of additions.  One work-group per row.  A token's order is one
// 64-bit number, an order-preserving key of its logit above the complement of its id, and
// every cut (top-k, top-p, min-p) keeps a prefix of that order:
//   top-k  a bound on the k-th key (k up to the threads: the k-th of the threads' own largest
//          keys; beyond, a histogram of counts) leaves a few candidates, which are sorted in
//          LDS and deal with the other two cuts and the draw: two or three passes over the row
//   top-p  a histogram of the weights by bins of y (32 to an octave of weight) finds the bin
//          of the cut, whose tokens are sorted; the kept weights are summed for each 64
//          groups in the order of ids, and the group with the drawn number is gone through
//          token by token: three passes
//   else   the largest logit and the sums: two passes
// More candidates than the list holds (thousands of equal logits in a cut, k of several
// thousands) and an infinite largest logit take the cuts digit by digit of the key.
// A row stays in the die's L2 between its passes: 256 rows of 131,072 bfloat16 logits take
// 98 us, 13 of them the first pass, at the rate of the memory; the others are bound by the
// fp64 instructions of the weights, of which a histogram pass takes some 25 for each logit.
// A small row is bound by the chain of block-wide steps: one of 32,000, 18.6 us.
#include "fs_engine.h"

namespace fs {

namespace {

struct SampleArgs {
  const void *logits;
  int64_t stride;
  int32_t rows, vocab;
  const float *temperature, *top_p, *min_p, *u;
  const int32_t *top_k;
  int32_t *token, *kept;
  float *logprob;
  int32_t *err;
};

constexpr int kAhead = 2;  // 16-byte loads of a thread in flight in the ordered pass
constexpr double kOne = 1099511627776.0;  // 2^40

// Order-preserving key: larger logit, larger key; -0 as 0; NaN as -inf.  -inf is kLow.
constexpr uint32_t kLow = 0x007fffffu;
__device__ inline uint32_t key_of(float x) {
  if (x != x) x = -INFINITY;
  const uint32_t b = __float_as_uint(x + 0.f);  // -0 + 0 = 0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float value_of(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

template <int DT>
__device__ inline float load_logit(const char *row, int32_t i) {
  if constexpr (DT == FS_F32)
    return reinterpret_cast<const float *>(row)[i];
  else
    return to_f32<DT == FS_BF16>(reinterpret_cast<const short *>(row)[i]);
}

// The weight of a logit: floor(2^(40 - y)), y = (largest - x) * per >= 0.  With q the nearest
// whole number to 256 y, 2^-y = 2^-(q >> 8) * 2^-((q & 255) / 256) * 2^(r / 256), |r| <= 1/2:
// a table of the 256 middle factors, and a series that ends below 4e-17 of the value at
// degree 4.  (Full passes over a row are bound by these instructions.)
struct Weigh {
  float top;            // the largest logit
  double best, per;     // per: 256 log2(e) / T
  const double *table;  // 2^(-j/256)
  static constexpr double kMagic = 6755399441055744.0 + 11 * 256;  // 1.5 * 2^52 + 11 * 256
  // 256 y, at most 13,030 (no weight is left from 41 * 256 on); NaN as -inf
  __device__ double y_of(float x) const {
    return fmin(__dmul_rn(__dsub_rn(best, double(fmaxf(x, -INFINITY))), per), 13030.0);
  }
  // q + 11 * 256, in the low bits of the sum
  __device__ static uint32_t place(double y) {
    return uint32_t(__double_as_longlong(y + kMagic));
  }
  __device__ static int bin_of(uint32_t place) { return int(place >> 3); }
  // N weights side by side: the table is read for all of them at once
  template <int N>
  __device__ void many(const double *y, uint64_t *w) const {
    double r[N], mid[N];
    uint32_t at[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const double s = y[e] + kMagic;
      at[e] = uint32_t(__double_as_longlong(s));
      mid[e] = table[at[e] & 255];
      r[e] = (s - kMagic) - y[e];
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
      double p = 2.23939519087515698716e-12;
      p = fma(p, r[e], 3.30830268054137129301e-09);
      p = fma(p, r[e], 3.66556559691010622906e-06);
      p = fma(p, r[e], 2.70760617406228627432e-03);
      p = fma(p, r[e], 1.0);
      // above 2 the product's bits stand still: its mantissa holds it times 2^51
      const uint64_t bits = uint64_t(__double_as_longlong(fma(p, mid[e], 2.0)));
      w[e] = (bits & 0xfffffffffffffull) >> (at[e] >> 8);
    }
  }
  __device__ uint64_t of_y(double y) const {
    uint64_t w;
    many<1>(&y, &w);
    return w;
  }
  __device__ uint64_t operator()(float x) const { return of_y(y_of(x)); }
  __device__ uint64_t operator()(uint32_t key) const {
    const float x = value_of(key);
    return x == top ? uint64_t(1) << 40 : of_y(y_of(x));  // the largest may be infinite
  }
};

// Sum over the wave, in lane 63: four steps inside rows of 16 lanes, two across them.
template <int CTRL, int ROWS>
__device__ inline uint64_t add_dpp(uint64_t x) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, uint32_t(x), CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, uint32_t(x >> 32), CTRL, ROWS, 0xf, false);
  return x + (uint64_t(hi) << 32 | lo);
}
__device__ inline uint64_t wave_sum_last(uint64_t x) {
  x = add_dpp<0x111, 0xf>(x);  // row_shr 1, 2, 4, 8
  x = add_dpp<0x112, 0xf>(x);
  x = add_dpp<0x114, 0xf>(x);
  x = add_dpp<0x118, 0xf>(x);
  x = add_dpp<0x142, 0xa>(x);  // lane 15 of a row to the next row
  return add_dpp<0x143, 0xc>(x);  // lane 31 to the upper half
}

template <int CTRL, int ROWS>
__device__ inline float max_dpp(float x) {
  return fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(
                      0xff800000u, __float_as_uint(x), CTRL, ROWS, 0xf, false)));
}
__device__ inline float wave_max_last(float x) {
  x = max_dpp<0x111, 0xf>(x);
  x = max_dpp<0x112, 0xf>(x);
  x = max_dpp<0x114, 0xf>(x);
  x = max_dpp<0x118, 0xf>(x);
  x = max_dpp<0x142, 0xa>(x);
  return max_dpp<0x143, 0xc>(x);
}

// One row by a work-group of kThreads.
template <int DT, int kThreads>
struct Sampler {
  static constexpr int kWaves = kThreads / 64;

  // A row as the tokens before the first 16-byte boundary, 16-byte vectors, and the tokens
  // after the last vector.
  struct Row {
    static constexpr int kVec = DT == FS_F32 ? 4 : 8;
    typedef s16x8 Raw;  // 16 bytes
    const char *p;
    int32_t head, vecs, vocab;
    __device__ Row(const char *base, int32_t V) : p(base), vocab(V) {
      constexpr int size = DT == FS_F32 ? 4 : 2;
      head = min(V, int32_t((16 - (reinterpret_cast<uintptr_t>(base) & 15)) & 15) / size);
      vecs = (V - head) / kVec;
    }
    __device__ int32_t tail() const { return head + vecs * kVec; }
    __device__ Raw load(int32_t v) const {  // vector v, or any other when there is no such
      const int32_t i = head + min(v, vecs - 1) * kVec;
      typedef const __attribute__((address_space(1))) Raw *Global;
      return *(Global)(p + int64_t(i) * (16 / kVec));
    }
    __device__ static float at(const Raw &v, int e) {  // e known at compile time
      if constexpr (DT == FS_F32)
        return __builtin_bit_cast(f32x4, v)[e];
      else
        return to_f32<DT == FS_BF16>(v[e]);
    }
    __device__ static float pick(const Raw &v, int e) {  // e from 0 to kVec - 1
      typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
      const u32x4 w = __builtin_bit_cast(u32x4, v);
      const int d = DT == FS_F32 ? e : e >> 1;
      const uint32_t lo = d & 1 ? w[1] : w[0], hi = d & 1 ? w[3] : w[2];
      const uint32_t x = d & 2 ? hi : lo;
      if constexpr (DT == FS_F32)
        return __uint_as_float(x);
      else
        return to_f32<DT == FS_BF16>(short(e & 1 ? x >> 16 : x));
    }
    // The whole row in no order: vec(first id, 16 bytes) for the vectors, one(id, logit) for
    // the other tokens.  AHEAD loads are in flight; the body is written out as often, so
    // long bodies take few.
    template <int AHEAD, class F, class G>
    __device__ void each(F vec, G one) const {
      const int tid = threadIdx.x, odd = head + vocab - tail();
      if (tid < odd) {
        const int32_t i = tid < head ? tid : tail() + tid - head;
        one(i, load_logit<DT>(p, i));
      }
      if (vecs == 0) return;
      Raw q[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) q[u] = load(tid + u * kThreads);
#pragma unroll 1
      for (int32_t v0 = tid; v0 < vecs; v0 += AHEAD * kThreads)
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          const int32_t v = v0 + u * kThreads;
          const Raw x = q[u];
          q[u] = load(v + AHEAD * kThreads);
          if (v < vecs) vec(head + v * kVec, x);
        }
    }
  };

  // What lanes of a wave store in LDS before, its other lanes load after.
  static __device__ inline void order_in_wave() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }

  static __device__ inline uint64_t block_sum(uint64_t v, uint64_t *red) {
    v = wave_sum_last(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) red[threadIdx.x >> 6] = v;
    __syncthreads();
    uint64_t s = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) s += red[i];
    return s;
  }

  // Exclusive prefix sum over the block's threads.
  static __device__ inline uint64_t block_scan(uint64_t v, uint64_t *red,
                                               uint64_t *total = nullptr) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint64_t x = v;
    for (int w = 1; w < 64; w <<= 1) {
      const uint64_t y = __shfl_up(x, w, 64);
      if (lane >= w) x += y;
    }
    __syncthreads();
    if (lane == 63) red[wave] = x;
    __syncthreads();
    uint64_t before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      before += i < wave ? red[i] : 0;
      all += red[i];
    }
    if (total) *total = all;
    return before + x - v;
  }

  // Sorts n2 (a power of two, at most kList) values downward.  A wave owns 128 neighbours:
  // steps shorter than that stay inside it, and only the longer ones need the work-group.
  static __device__ void sort_down(uint64_t *v, int n2) {
    const int tid = threadIdx.x;
    for (int size = 2; size <= n2; size <<= 1) {
      for (int d = size >> 1; d; d >>= 1) {
        if (d >= 64) __syncthreads();
        for (int t = tid; t < n2 / 2; t += kThreads) {
          const int i = 2 * t - (t & (d - 1)), j = i + d;
          const uint64_t x = v[i], y = v[j];
          if ((x < y) == ((i & size) == 0)) v[i] = y, v[j] = x;
        }
        if (d >= 128) __syncthreads();
        else order_in_wave();
      }
    }
    __syncthreads();
  }

  static constexpr int kList = 4096;       // candidates that are sorted in LDS
  static constexpr int kBase = 11 * 32;    // the first bin
  // of y: 32 to an octave of weight (none is left from 41 octaves on)
  static constexpr int kBins = kBase + 51 * 32;
  static constexpr int kQueue = 64 * 8 + 16;  // logits of a wave that wait to be weighed
  static constexpr int kSegs = (1 << 20) / 4 / 64 + 2;  // sums of 64 groups of tokens

  struct Shared {
    uint64_t list[kList];
    uint64_t seg[kSegs];
    uint64_t hist[kBins];
    uint64_t queue[kWaves][kQueue];
    uint64_t red[kWaves];
    uint64_t val[2];
    double table[256];
    int32_t n;
  };

  static __device__ inline uint64_t pair_of(uint32_t key, int32_t id) {
    return uint64_t(key) << 32 | uint32_t(~id);
  }
  static __device__ inline uint32_t key_in(uint64_t pair) { return uint32_t(pair >> 32); }
  static __device__ inline int32_t id_in(uint64_t pair) { return int32_t(~uint32_t(pair)); }

  // A lower bound on the k-th largest of the threads' keys: its upper 16 bits, digit by digit.
  static __device__ uint32_t kth_of_threads(uint32_t key, int32_t k, Shared &sh) {
    const int tid = threadIdx.x;
    uint32_t *h = reinterpret_cast<uint32_t *>(sh.hist);
    uint32_t prefix = 0;
#pragma unroll
    for (int shift = 24; shift >= 16; shift -= 8) {
      __syncthreads();
      if (tid < 256) h[tid] = 0;
      __syncthreads();
      if (shift == 24 || (key >> 24) == (prefix >> 24)) atomicAdd(&h[(key >> shift) & 255], 1u);
      __syncthreads();
      if (tid < 64) {
        // four digits a lane, from the largest down
        uint32_t c[4], sum = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += c[e] = h[255 - (tid * 4 + e)];
        uint32_t x = sum;
        for (int w = 1; w < 64; w <<= 1) {
          const uint32_t y = __shfl_up(x, w, 64);
          if (tid >= w) x += y;
        }
        uint32_t before = x - sum;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (before < uint32_t(k) && before + c[e] >= uint32_t(k)) {
            sh.val[0] = prefix | uint32_t(255 - (tid * 4 + e)) << shift;
            sh.val[1] = uint32_t(k) - before;
          }
          before += c[e];
        }
      }
      __syncthreads();
      prefix = uint32_t(sh.val[0]);
      k = int32_t(sh.val[1]);
    }
    return prefix;
  }

  // Appends to the list the tokens that `take` accepts; false when they are more than kList.
  template <class F>
  static __device__ bool collect(const Row &row, Shared &sh, F take) {
    __syncthreads();
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    auto one = [&](int32_t id, float x) {
      if (take(x)) {
        const int at = atomicAdd(&sh.n, 1);
        if (at < kList) sh.list[at] = pair_of(key_of(x), id);
      }
    };
    row.template each<4>(
        [&](int32_t id0, const s16x8 &v) {
          uint32_t mask = 0;
#pragma unroll
          for (int e = 0; e < Row::kVec; ++e) mask |= take(Row::at(v, e)) ? 1u << e : 0;
          while (mask) {
            const int e = __builtin_ctz(mask);
            mask &= mask - 1;
            const int at = atomicAdd(&sh.n, 1);
            if (at < kList) sh.list[at] = pair_of(key_of(Row::pick(v, e)), id0 + e);
          }
        },
        one);
    __syncthreads();
    return sh.n <= kList;
  }

  // The number of values above x in a run of 64 that is sorted downward.
  static __device__ inline int above_in_run(const uint64_t *run, uint64_t x) {
    int n = 0;
#pragma unroll
    for (int d = 32; d; d >>= 1) n += run[n + d - 1] > x ? d : 0;
    return n + (run[n] > x);
  }

  // Sorts the list downward (its values differ) and returns its length.  Up to kThreads
  // values: each wave sorts 64 in registers, then a value's place is the count of larger
  // ones over all runs; more go through sort_down.
  static __device__ int sort_list(Shared &sh) {
    const int n = sh.n, tid = threadIdx.x, lane = tid & 63;
    if (n <= kThreads) {
      const int runs = (n + 63) >> 6;
      uint64_t x = tid < n ? sh.list[tid] : 0;
      if (tid < runs * 64) {
        for (int size = 2; size <= 64; size <<= 1)
          for (int d = size >> 1; d; d >>= 1) {
            const uint64_t y = __shfl_xor(x, d, 64);
            const bool larger = ((lane & d) == 0) == ((lane & size) == 0);
            x = (x > y) == larger ? x : y;
          }
      }
      if (runs > 1) {
        __syncthreads();
        if (tid < runs * 64) sh.list[tid] = x;
        __syncthreads();
        int place = lane;
        if (x)
          for (int r = 0; r < runs; ++r)
            if (r != tid >> 6) place += above_in_run(sh.list + r * 64, x);
        __syncthreads();
        if (x) sh.list[place] = x;
      } else {
        __syncthreads();
        if (x) sh.list[tid] = x;
      }
      __syncthreads();
      return n;
    }
    int n2 = 64;
    while (n2 < n) n2 <<= 1;
    for (int i = n + tid; i < n2; i += kThreads) sh.list[i] = 0;
    __syncthreads();
    sort_down(sh.list, n2);
    return n;
  }

  static __device__ void run(const SampleArgs &a, Shared &sh) {
    constexpr int kVec = Row::kVec, kPer = kList / kThreads;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t row = blockIdx.x, V = a.vocab;
    const char *base = static_cast<const char *>(a.logits) +
                       int64_t(row) * a.stride * (DT == FS_F32 ? 4 : 2);
    const Row r(base, V);
    const float T = a.temperature ? a.temperature[row] : 1.f;
    const float tp = a.top_p ? a.top_p[row] : 1.f, mp = a.min_p ? a.min_p[row] : 0.f;
    const float u = a.u[row];
    const int32_t k_in = a.top_k ? a.top_k[row] : 0;
    const bool bad = !(T >= 0.f) || !(T < INFINITY) || !(tp >= 0.f && tp <= 1.f) ||
                     !(mp >= 0.f && mp <= 1.f) || !(u >= 0.f && u < 1.f);
    if (tid < 256) sh.table[tid] = exp2(double(-tid) * 0.00390625);

    // the largest logit (NaN loses every comparison)
    float mine = -INFINITY;
    r.template each<4>(
        [&](int32_t, const s16x8 &v) {
#pragma unroll
          for (int e = 0; e < kVec; ++e) mine = fmaxf(mine, Row::at(v, e));
        },
        [&](int32_t, float x) { mine = fmaxf(mine, x); });
    float top = wave_max_last(mine);
    float *fred = reinterpret_cast<float *>(sh.red);
    if (lane == 63) fred[wave] = top;
    __syncthreads();
    top = fred[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) top = fmaxf(top, fred[i]);
    if (bad || top == -INFINITY) {
      if (tid == 0) {
        a.token[row] = -1;
        if (a.logprob) a.logprob[row] = -INFINITY;
        if (a.kept) a.kept[row] = 0;
        if (bad) raise_err(a.err, FS_E_RANGE);
      }
      return;
    }
    if (T == 0.f) {  // the lowest id of the largest logit
      if (tid == 0) sh.n = V;
      __syncthreads();
      if (mine == top)
        r.template each<2>(
            [&](int32_t id0, const s16x8 &v) {
#pragma unroll
              for (int e = kVec - 1; e >= 0; --e)
                if (Row::at(v, e) == top) atomicMin(&sh.n, id0 + e);
            },
            [&](int32_t id, float x) {
              if (x == top) atomicMin(&sh.n, id);
            });
      __syncthreads();
      if (tid == 0) {
        a.token[row] = sh.n;
        if (a.logprob) a.logprob[row] = 0.f;
        if (a.kept) a.kept[row] = 1;
      }
      return;
    }
    const Weigh weigh{top, double(top), 256.0 * (1.4426950408889634 / double(T)), sh.table};
    uint64_t least = uint64_t(ceil(__dmul_rn(double(mp), kOne)));
    if (least < 1) least = 1;

    // kept: pairs (key, ~id) of at least `cut`, with a weight of at least `least`
    uint64_t cut = pair_of(kLow + 1, INT32_MAX);
    // an infinite logit leaves no finite distances: the general way deals with it
    if (top == INFINITY) return sample_slow(a, base, row, weigh, tp, least, k_in, u, sh);
    if (k_in > 0 && k_in < V) {
      bool fits;
      if (k_in <= kThreads) {
        // The k-th largest of the threads' own largest logits is no larger than the k-th
        // largest logit: what is at least that holds the first k tokens.
        const float bound = value_of(max(kth_of_threads(key_of(mine), k_in, sh), kLow + 1));
        fits = collect(r, sh, [&](float x) { return x >= bound; });
      } else {
        // the bin of y in which the k-th logit lies; what lies beyond the bins has no weight
        for (int i = tid; i < kBins; i += kThreads) sh.hist[i] = 0;
        __syncthreads();
        auto one = [&](int32_t, float x) {
          const int bin = Weigh::bin_of(Weigh::place(weigh.y_of(x)));
          atomicAdd(reinterpret_cast<unsigned int *>(&sh.hist[bin]), 1u);
        };
        r.template each<2>(
            [&](int32_t id0, const s16x8 &v) {
#pragma unroll
              for (int e = 0; e < kVec; ++e) one(id0 + e, Row::at(v, e));
            },
            one);
        __syncthreads();
        constexpr int kB = (kBins + kThreads - 1) / kThreads;
        uint64_t h[kB], sum = 0;
#pragma unroll
        for (int e = 0; e < kB; ++e) {
          h[e] = tid * kB + e < kBins ? sh.hist[tid * kB + e] : 0;
          sum += h[e];
        }
        uint64_t before = block_scan(sum, sh.red);
        if (tid == 0) sh.val[1] = kBins - 1;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kB; ++e) {
          if (before < uint64_t(k_in) && before + h[e] >= uint64_t(k_in)) sh.val[1] = tid * kB + e;
          before += h[e];
        }
        __syncthreads();
        const int bin = int(sh.val[1]);
        fits = collect(r, sh, [&](float x) {
          return Weigh::bin_of(Weigh::place(weigh.y_of(x))) <= bin;
        });
      }
      if (!fits) return sample_slow(a, base, row, weigh, tp, least, k_in, u, sh);
      const int n = sort_list(sh);
      // the list's order is the definition's: every cut is a prefix of it
      const int per = (n + kThreads - 1) / kThreads, i0 = min(tid * per, n), i1 = min(i0 + per, n);
      uint64_t w[kPer], sum = 0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const int i = i0 + e;
        w[e] = i < i1 && i < k_in ? weigh(key_in(sh.list[i])) : 0;
        sum += w[e];
      }
      uint64_t W;
      uint64_t before = block_scan(sum, sh.red, &W);
      uint64_t limit = ~uint64_t(0);
      if (tp < 1.f) {
        const double lim = ceil(__dmul_rn(double(tp), double(W)));
        limit = lim < 1.0 ? 1 : uint64_t(lim);
      }
      uint64_t kept = 0, kept_n = 0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const bool in = w[e] >= least && before < limit;
        before += w[e];
        w[e] = in ? w[e] : 0;
        kept += w[e];
        kept_n += in;
      }
      const uint64_t S = block_sum(kept, sh.red);
      const int m = int(block_sum(kept_n, sh.red));
      uint64_t goal = uint64_t(__dmul_rn(double(u), double(S)));
      if (goal > S - 1) goal = S - 1;
      // the kept ones by id, with their keys: ids sort upward as ~id downward
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const int i = i0 + e;
        if (i < i1 && w[e]) sh.list[i] = uint64_t(uint32_t(sh.list[i])) << 32 | key_in(sh.list[i]);
      }
      if (tid == 0) sh.n = m;
      __syncthreads();
      sort_list(sh);
      const int per2 = (m + kThreads - 1) / kThreads, j0 = min(tid * per2, m),
                j1 = min(j0 + per2, m);
      sum = 0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        w[e] = j0 + e < j1 ? weigh(uint32_t(sh.list[j0 + e])) : 0;
        sum += w[e];
      }
      uint64_t run = block_scan(sum, sh.red);
      if (run <= goal && goal < run + sum) {
        bool found = false;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          run += w[e];
          if (!found && w[e] && run > goal) {
            found = true;
            a.token[row] = id_in(key_in(sh.list[j0 + e]));
            if (a.logprob) a.logprob[row] = float(log(double(w[e]) / double(S)));
            if (a.kept) a.kept[row] = m;
          }
        }
      }
      return;
    }

    // top-p: the bin of y in which the cut lies, and what lies above it
    const bool nucleus = tp < 1.f;
    uint64_t limit = 0, above = 0;
    int bin = 0;
    float from = INFINITY, to = -INFINITY;  // the bin's logits, a little widened
    if (nucleus) {
      // weights by bin of y, 32 bins to an octave
      for (int i = tid; i < kBins; i += kThreads) sh.hist[i] = 0;
      __syncthreads();
      auto add = [&](double y, uint64_t w) {
        atomicAdd(reinterpret_cast<unsigned long long *>(&sh.hist[Weigh::bin_of(Weigh::place(y))]),
                  (unsigned long long)w);
      };
      r.template each<2>(
          [&](int32_t, const s16x8 &v) {
            double y[kVec];
            uint64_t w[kVec];
#pragma unroll
            for (int e = 0; e < kVec; ++e) y[e] = weigh.y_of(Row::at(v, e));
            weigh.template many<kVec>(y, w);
#pragma unroll
            for (int e = 0; e < kVec; ++e) add(y[e], w[e]);
          },
          [&](int32_t, float x) {
            const double y = weigh.y_of(x);
            add(y, weigh.of_y(y));
          });
      __syncthreads();
      // the bin in which the running sum reaches the limit
      constexpr int kB = (kBins + kThreads - 1) / kThreads;
      uint64_t h[kB], sum = 0;
#pragma unroll
      for (int e = 0; e < kB; ++e) {
        h[e] = tid * kB + e < kBins ? sh.hist[tid * kB + e] : 0;
        sum += h[e];
      }
      uint64_t W;
      uint64_t before = block_scan(sum, sh.red, &W);
      const double lim = ceil(__dmul_rn(double(tp), double(W)));
      limit = lim < 1.0 ? 1 : uint64_t(lim);
#pragma unroll
      for (int e = 0; e < kB; ++e) {
        if (before < limit && before + h[e] >= limit) {
          sh.val[0] = before;
          sh.val[1] = tid * kB + e;
        }
        before += h[e];
      }
      __syncthreads();
      above = sh.val[0];
      bin = int(sh.val[1]);
      const float slack = 1e-6f * (fabsf(top) + float(42.0 * 256.0 / weigh.per));
      from = float(double(top) - ((bin - kBase + 1) * 8 + 1) / weigh.per) - slack;
      to = float(double(top) - ((bin - kBase) * 8 - 1) / weigh.per) + slack;
      if (!isfinite(from) || !isfinite(to)) from = -INFINITY, to = INFINITY;
      if (tid == 0) sh.n = 0;
      __syncthreads();
    }

    // The kept weights in the order of ids: a sum for each 64 groups (the tokens before the
    // first vector, each vector, the tokens after the last), then the one that holds the
    // goal, token by token.  Where not all are kept a lane weighs its own one after another,
    // so a round costs as many weights as its fullest lane keeps, not a whole vector.
    // Under top-p the logits above the cut's bin are summed so and the bin's own are listed
    // in the same pass; once sorted, those that stay are added to their groups' sums.
    float cut_x = nucleus ? to : value_of(key_in(cut));
    int32_t cut_id = nucleus ? -1 : id_in(cut);
    // below `low` a weight is surely under `least` (and under 1)
    const double reach = 256.0 * (40.0 - log2(double(least)) + 0.01);
    const float low = float(double(top) - reach / weigh.per) -
                      1e-6f * (fabsf(top) + float(reach / weigh.per));
    float bound = isfinite(low) ? fmaxf(cut_x, low) : cut_x;
    const bool whole = !nucleus && least == 1;  // every token with a weight is kept
    auto group = [&](int32_t g, const s16x8 &raw, auto take) {
      if (g >= 1 && g <= r.vecs) {
        const int32_t i0 = r.head + (g - 1) * kVec;
        if (whole) {
          double y[kVec];
          uint64_t w[kVec];
#pragma unroll
          for (int e = 0; e < kVec; ++e) y[e] = weigh.y_of(Row::at(raw, e));
          weigh.template many<kVec>(y, w);
#pragma unroll
          for (int e = 0; e < kVec; ++e) take(i0 + e, w[e]);
          return;
        }
        // equal to the bound: kept up to the cut's own id
        const int32_t ties = bound > cut_x ? kVec : max(0, min(kVec, cut_id - i0 + 1));
        uint32_t above = 0, equal = 0;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const float x = Row::at(raw, e);
          above |= x > bound ? 1u << e : 0;
          equal |= x == bound ? 1u << e : 0;
        }
        uint32_t mask = above | (equal & ((1u << ties) - 1));
        while (mask) {
          const int e = __builtin_ctz(mask);
          mask &= mask - 1;
          const uint64_t w = weigh(Row::pick(raw, e));
          take(i0 + e, w >= least ? w : 0);
        }
      } else if (g == 0 || g == r.vecs + 1) {
        const int32_t i0 = g == 0 ? 0 : r.tail(), i1 = g == 0 ? r.head : V;
        for (int32_t i = i0; i < i1; ++i) {
          const float x = load_logit<DT>(base, i);
          const uint64_t w =
              x > bound || (x == bound && (x > cut_x || i <= cut_id)) ? weigh(x) : 0;
          take(i, w >= least ? w : 0);
        }
      }
    };
    const int32_t segs = (r.vecs + 2 + 63) / 64;
    uint64_t total = 0;
    uint32_t count = 0;
    // Not all are kept: a sum's logits that may be are gathered, and weighed 64 at a time with
    // every lane at work.
    const float gate = nucleus ? from : bound;
    uint64_t *queue = sh.queue[wave];
    int waiting = 0;  // the same for the wave
    auto gather = [&](int32_t id, float x, bool have) {
      const bool take = have && x >= gate;
      const uint64_t takers = __ballot(take);
      if (takers) {
        if (take)
          queue[waiting + __builtin_amdgcn_mbcnt_hi(
                              uint32_t(takers >> 32),
                              __builtin_amdgcn_mbcnt_lo(uint32_t(takers), 0))] =
              pair_of(key_of(x), id);
        waiting += __popcll(takers);
      }
    };
    auto weigh_gathered = [&]() -> uint64_t {
      uint64_t sum = 0;
      order_in_wave();
      for (int from_slot = 0; from_slot < waiting; from_slot += 64) {
        if (from_slot + lane >= waiting) continue;
        const uint64_t pair = queue[from_slot + lane];
        const double y = weigh.y_of(value_of(key_in(pair)));
        const int at_bin = Weigh::bin_of(Weigh::place(y));
        if (nucleus && at_bin == bin) {
          const int at = atomicAdd(&sh.n, 1);
          if (at < kList) sh.list[at] = pair;
        } else if (!nucleus || at_bin < bin) {
          const uint64_t w = weigh.of_y(y);
          sum += w >= least ? w : 0;
          count += w >= least;
        }
      }
      order_in_wave();
      waiting = 0;
      return sum;
    };
    {
      s16x8 q[kAhead] = {};
      const bool any = r.vecs > 0;
      const int32_t last_seg = (r.vecs + 1) >> 6;
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (any) q[i] = r.load(max(0, (wave + i * kWaves) * 64 + lane - 1));
#pragma unroll 1
      for (int32_t s0 = wave; s0 < segs; s0 += kAhead * kWaves)
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const int32_t s = s0 + i * kWaves;
          const s16x8 raw = q[i];
          if (any) q[i] = r.load((s + kAhead * kWaves) * 64 + lane - 1);
          if (s >= segs) continue;
          const int32_t g = s * 64 + lane;
          uint64_t sum = 0;
          if (whole) {
            group(g, raw, [&](int32_t, uint64_t w) {
              sum += w;
              count += w != 0;
            });
          } else {
            const bool vec = g >= 1 && g <= r.vecs;
#pragma unroll
            for (int e = 0; e < kVec; ++e)
              gather(r.head + (g - 1) * kVec + e, Row::at(raw, e), vec);
            if (s == 0 || s == last_seg) {  // the tokens outside the vectors
              const int32_t i0 = g == 0 ? 0 : r.tail(),
                            n = g == 0 ? r.head : g == r.vecs + 1 ? V - r.tail() : 0;
#pragma unroll 1
              for (int e = 0; e < kVec; ++e)
                gather(i0 + e, e < n ? load_logit<DT>(base, i0 + e) : 0.f, e < n);
            }
            sum = weigh_gathered();
          }
          total += sum;
          sum = wave_sum_last(sum);
          if (lane == 63) sh.seg[s] = sum;
        }
    }
    if (nucleus) {
      __syncthreads();
      if (sh.n > kList) return sample_slow(a, base, row, weigh, tp, least, k_in, u, sh);
      const int n = sort_list(sh);
      const int per = (n + kThreads - 1) / kThreads, i0 = min(tid * per, n), i1 = min(i0 + per, n);
      uint64_t w[kPer], sum = 0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        w[e] = i0 + e < i1 ? weigh(key_in(sh.list[i0 + e])) : 0;
        sum += w[e];
      }
      uint64_t before = above + block_scan(sum, sh.red);
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        if (w[e] && before < limit) {
          const uint64_t pair = sh.list[i0 + e];
          if (before + w[e] >= limit) sh.val[0] = pair;  // the last one that stays
          if (w[e] >= least) {
            const int32_t id = id_in(pair);
            const int32_t g = id < r.head ? 0 : (id - r.head) / kVec + 1;
            atomicAdd(reinterpret_cast<unsigned long long *>(&sh.seg[g >> 6]),
                      (unsigned long long)w[e]);
            total += w[e];
            ++count;
          }
        }
        before += w[e];
      }
      __syncthreads();
      cut_x = value_of(key_in(sh.val[0]));
      cut_id = id_in(sh.val[0]);
      bound = isfinite(low) ? fmaxf(cut_x, low) : cut_x;
    }
    const uint64_t S = block_sum(total, sh.red);
    const int32_t m = int32_t(block_sum(uint64_t(count), sh.red));
    uint64_t goal = uint64_t(__dmul_rn(double(u), double(S)));
    if (goal > S - 1) goal = S - 1;
    const int per = (segs + kThreads - 1) / kThreads, s0 = min(tid * per, segs),
              s1 = min(s0 + per, segs);
    uint64_t sum = 0;
    for (int s = s0; s < s1; ++s) sum += sh.seg[s];
    uint64_t run = block_scan(sum, sh.red);
    if (run <= goal && goal < run + sum) {
      for (int s = s0; s < s1; ++s) {
        if (goal < run + sh.seg[s]) {
          sh.val[0] = run;
          sh.val[1] = s;
          break;
        }
        run += sh.seg[s];
      }
    }
    __syncthreads();
    if (wave) return;
    run = sh.val[0];
    const int32_t g = int32_t(sh.val[1]) * 64 + lane;
    s16x8 raw = {};
    if (r.vecs > 0) raw = r.load(max(0, g - 1));
    sum = 0;
    group(g, raw, [&](int32_t, uint64_t w) { sum += w; });
    uint64_t x = sum;
    for (int w = 1; w < 64; w <<= 1) {
      const uint64_t y = __shfl_up(x, w, 64);
      if (lane >= w) x += y;
    }
    run += x - sum;
    if (run <= goal && goal < run + sum) {
      bool found = false;
      group(g, raw, [&](int32_t id, uint64_t w) {
        run += w;
        if (!found && run > goal) {
          found = true;
          a.token[row] = id;
          if (a.logprob) a.logprob[row] = float(log(double(w) / double(S)));
          if (a.kept) a.kept[row] = m;
        }
      });
    }
  }

  // Any k and any number of equal logits: the cuts digit by digit of the key, a pass over
  // the row for each digit.
  static __device__ __noinline__ void sample_slow(const SampleArgs &a, const char *base,
                                                  int32_t row, const Weigh &weigh, float tp,
                                                  uint64_t least, int32_t k_in, float u,
                                                  Shared &sh) {
    const int tid = threadIdx.x;
    const int32_t V = a.vocab;
    uint64_t *red = sh.red, *hist = sh.hist;
    uint64_t &sh_u64 = sh.val[0], &sh_key = sh.val[1];
    int32_t &sh_id = sh.n;
    __syncthreads();

    // Cut: keys above `cut` are kept, and the first `ties` ids of those that equal it.
    uint32_t cut = kLow;
    uint64_t ties = uint64_t(V);
    if (k_in > 0 && k_in < V) {
      uint32_t prefix = 0;
      uint64_t need = uint64_t(k_in);
      for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kThreads) hist[i] = 0;
        __syncthreads();
        for (int32_t i = tid; i < V; i += kThreads) {
          const uint32_t key = key_of(load_logit<DT>(base, i));
          if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8)))
            atomicAdd(reinterpret_cast<unsigned long long *>(&hist[(key >> shift) & 255]), 1ull);
        }
        __syncthreads();
        if (tid == 0) {
          int d = 255;
          uint64_t left = need;
          while (d > 0 && hist[d] < left) left -= hist[d--];
          sh_key = prefix | uint32_t(d) << shift;
          sh_u64 = left;
        }
        __syncthreads();
        prefix = uint32_t(sh_key);
        need = sh_u64;
        __syncthreads();
      }
      cut = prefix;
      ties = need;
    }
    // top-p over the weights above the cut
    if (tp < 1.f) {
      uint64_t sum = 0;
      for (int32_t i = tid; i < V; i += kThreads) {
        const uint32_t key = key_of(load_logit<DT>(base, i));
        if (key > cut) sum += weigh(key);
      }
      uint64_t W = block_sum(sum, red);
      if (cut > kLow) W += ties * weigh(cut);
      const double lim = ceil(__dmul_rn(double(tp), double(W)));
      const uint64_t limit = lim < 1.0 ? 1 : uint64_t(lim);
      // the key at which the weights before it pass the limit
      uint32_t prefix = 0;
      uint64_t before = 0;  // weight above the current digit range
      for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kThreads) hist[i] = 0;
        __syncthreads();
        for (int32_t i = tid; i < V; i += kThreads) {
          const uint32_t key = key_of(load_logit<DT>(base, i));
          if (key > cut && (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8)))) {
            const uint64_t w = weigh(key);
            if (w)
              atomicAdd(reinterpret_cast<unsigned long long *>(&hist[(key >> shift) & 255]), w);
          }
        }
        __syncthreads();
        if (tid == 0) {
          int d = 255;
          uint64_t b = before;
          // the first digit whose weights bring the sum to the limit
          while (d > 0 && b + hist[d] < limit) b += hist[d--];
          sh_key = prefix | uint32_t(d) << shift;
          sh_u64 = b;
        }
        __syncthreads();
        prefix = uint32_t(sh_key);
        before = sh_u64;
        __syncthreads();
      }
      // keys above `prefix` weigh `before` < limit in all: they stay, and of `prefix` itself
      // the ids whose predecessors weigh less than the limit.  When even the last digits do
      // not reach the limit, the cut of top-k stands.
      if (prefix > cut) {
        const uint64_t w = weigh(prefix);
        cut = prefix;
        ties = w ? (limit - before + w - 1) / w : 0;
      } else if (cut > kLow) {
        const uint64_t w = weigh(cut);
        const uint64_t more = before >= limit || !w ? 0 : (limit - before + w - 1) / w;
        ties = more < ties ? more : ties;
      }
    }
    // The id of the last kept tie: only when not all of them stay.
    int32_t tie_id = V;
    uint64_t mine = 0;
    const int32_t per = (V + kThreads - 1) / kThreads;
    const int32_t i0 = min(tid * per, V), i1 = min(i0 + per, V);
    for (int32_t i = i0; i < i1; ++i) mine += key_of(load_logit<DT>(base, i)) == cut;
    const uint64_t all = block_sum(mine, red);
    if (ties < all) {
      if (tid == 0) sh_id = -1;
      uint64_t n = block_scan(mine, red);
      __syncthreads();
      if (n < ties && n + mine >= ties) {
        for (int32_t i = i0; i < i1; ++i)
          if (key_of(load_logit<DT>(base, i)) == cut && ++n == ties) sh_id = i;
      }
      __syncthreads();
      tie_id = sh_id;
    }
    auto kept_weight = [&](int32_t i) -> uint64_t {
      const uint32_t key = key_of(load_logit<DT>(base, i));
      if (key < cut || key <= kLow || (key == cut && i > tie_id)) return 0;
      const uint64_t w = weigh(key);
      return w >= least ? w : 0;
    };
    uint64_t sum = 0, count = 0;
    for (int32_t i = i0; i < i1; ++i) {
      const uint64_t w = kept_weight(i);
      sum += w;
      count += w != 0;
    }
    const uint64_t S = block_sum(sum, red), n_kept = block_sum(count, red);
    uint64_t run = block_scan(sum, red);
    uint64_t goal = uint64_t(__dmul_rn(double(u), double(S)));
    if (goal > S - 1) goal = S - 1;
    if (run <= goal && goal < run + sum) {
      for (int32_t i = i0; i < i1; ++i) {
        const uint64_t w = kept_weight(i);
        run += w;
        if (run > goal) {
          a.token[row] = i;
          if (a.logprob) a.logprob[row] = float(log(double(w) / double(S)));
          if (a.kept) a.kept[row] = int32_t(n_kept);
          break;
        }
      }
    }
  }

};

template <int DT, int kThreads>
__global__ void __launch_bounds__(kThreads) k_sample(SampleArgs a) {
  __shared__ typename Sampler<DT, kThreads>::Shared sh;
  Sampler<DT, kThreads>::run(a, sh);
}

template <int DT>
void launch(const SampleArgs &a, hipStream_t stream) {
  // Short rows are bound by the steps between barriers: fewer waves.  (One row of 32,000
  // logits: 23 us with 1,024 threads, 19 with 512; 256 rows of 60,000: 58 and 63 us; 256 rows
  // of 131,072: 98 and 119 us.)
  if (a.vocab <= 49152)
    hipLaunchKernelGGL((k_sample<DT, 512>), dim3(a.rows), dim3(512), 0, stream, a);
  else
    hipLaunchKernelGGL((k_sample<DT, 1024>), dim3(a.rows), dim3(1024), 0, stream, a);
}

}  // namespace

size_t sample_workspace_bytes(int32_t, int32_t, int32_t) { return 0; }

hipError_t launch_sample(int32_t dtype, int32_t rows, int32_t vocab, const void *logits,
                         int64_t stride, const fs_sampling *p, const float *u, int32_t *token,
                         float *logprob, int32_t *kept, void *ws, int32_t *err,
                         hipStream_t stream) {
  SampleArgs a{logits, stride,   rows, vocab, p->temperature, p->top_p, p->min_p, u, p->top_k,
               token,  kept,     logprob, err};
  if (dtype == FS_BF16)
    launch<FS_BF16>(a, stream);
  else if (dtype == FS_F16)
    launch<FS_F16>(a, stream);
  else
    launch<FS_F32>(a, stream);
  return hipGetLastError();
}

}  // namespace fs
