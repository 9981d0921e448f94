// The next token of each row from its logits and one given random number, in whole-number
// weights (2^40 for the largest logit): every sum is exact, so the kept set and the token
// do not depend on the order of additions.  One work-group per row.  A token's order is one
// 64-bit number, an order-preserving key of its logit above the complement of its id, and
// every cut (top-k, top-p, min-p) keeps a prefix of that order:
//   top-k  a bound on the k-th key leaves a few candidates, which are sorted in LDS
//   top-p  a histogram of the weights over the logits finds the bin of the cut, and the
//          tokens of that bin are sorted
//   then the kept weights are summed in the order of ids up to the drawn number.
// More candidates than the list holds (k above 1,024, thousands of equal logits) take the
// cuts digit by digit of the key instead.
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

constexpr int kThreads = 1024;
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

// A row as groups of consecutive tokens: the ones before the first 16-byte boundary, the
// 16-byte vectors, the ones after the last vector.
template <int DT>
struct Row {
  static constexpr int kVec = DT == FS_F32 ? 4 : 8;
  const char *p;
  int32_t head, vecs, vocab;
  __device__ Row(const char *base, int32_t V) : p(base), vocab(V) {
    constexpr int size = DT == FS_F32 ? 4 : 2;
    head = min(V, int32_t((16 - (reinterpret_cast<uintptr_t>(base) & 15)) & 15) / size);
    vecs = (V - head) / kVec;
  }
  __device__ int32_t groups() const { return vecs + 2; }
  // f(id, logit) for the tokens of a group, in order
  template <class F>
  __device__ void visit(int32_t g, F f) const {
    if (g >= 1 && g <= vecs) {
      const int32_t i0 = head + (g - 1) * kVec;
      if constexpr (DT == FS_F32) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(p + int64_t(i0) * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) f(i0 + e, v[e]);
      } else {
        const s16x8 v = *reinterpret_cast<const s16x8 *>(p + int64_t(i0) * 2);
#pragma unroll
        for (int e = 0; e < 8; ++e) f(i0 + e, to_f32<DT == FS_BF16>(v[e]));
      }
    } else if (g < groups()) {
      const int32_t i0 = g == 0 ? 0 : head + vecs * kVec, i1 = g == 0 ? head : vocab;
      for (int32_t i = i0; i < i1; ++i) f(i, load_logit<DT>(p, i));
    }
  }
};

// 2^-y for y >= 0 times 2^40, rounded down.  2^f for |f| <= 1/2 by the Taylor series of
// exp(f ln 2) (degree 12: below 2e-16 of the value).
__device__ inline uint64_t weight_of(double y) {
  const double k = rint(-y), z = (-y - k) * 0.693147180559945309417;
  double p = 2.08767569878680989792e-9;  // 1/12!
  p = fma(p, z, 2.50521083854417187751e-8);
  p = fma(p, z, 2.75573192239858906526e-7);
  p = fma(p, z, 2.75573192239858906526e-6);
  p = fma(p, z, 2.48015873015873015873e-5);
  p = fma(p, z, 1.98412698412698412698e-4);
  p = fma(p, z, 1.38888888888888888889e-3);
  p = fma(p, z, 8.33333333333333333333e-3);
  p = fma(p, z, 4.16666666666666666667e-2);
  p = fma(p, z, 1.66666666666666666667e-1);
  p = fma(p, z, 0.5);
  p = fma(p, z, 1.0);
  p = fma(p, z, 1.0);
  // a whole number below 2^52 lies in the low bits of its sum with 2^52
  const double w = floor(ldexp(p, int(k) + 40)) + 4503599627370496.0;
  return y < 41.0 ? uint64_t(__double_as_longlong(w)) & ((uint64_t(1) << 52) - 1) : 0;
}

struct Weigh {
  uint32_t top;  // key of the largest logit
  double best, per;
  // the exponent: weight 2^(40 - y); 0 for the largest logit, whatever it is
  __device__ double y_of(uint32_t key) const {
    return key == top ? 0.0 : __dmul_rn(__dsub_rn(best, double(value_of(key))), per);
  }
  __device__ uint64_t operator()(uint32_t key) const { return weight_of(y_of(key)); }
};

template <class T>
__device__ T block_sum(T v, T *red) {
  for (int w = 32; w; w >>= 1) v += __shfl_xor(v, w, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  T s = 0;
  for (int i = 0; i < kThreads / 64; ++i) s += red[i];
  return s;
}

// Exclusive prefix sum over the block's threads.
__device__ inline uint64_t block_scan(uint64_t v, uint64_t *red) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t x = v;
  for (int w = 1; w < 64; w <<= 1) {
    const uint64_t y = __shfl_up(x, w, 64);
    if (lane >= w) x += y;
  }
  __syncthreads();
  if (lane == 63) red[wave] = x;
  __syncthreads();
  uint64_t before = 0;
  for (int i = 0; i < wave; ++i) before += red[i];
  return before + x - v;
}

// Sorts n2 (a power of two, at most kList) values downward.  A wave owns 128 neighbours:
// steps shorter than that stay inside it, and only the longer ones need the work-group.
__device__ void sort_down(uint64_t *v, int n2) {
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
      else __builtin_amdgcn_wave_barrier();
    }
  }
  __syncthreads();
}

constexpr int kList = 4096;       // candidates that are sorted in LDS
constexpr int kBins = 41 * 32;    // of y: 32 to an octave of weight
constexpr int kSegs = (1 << 20) / 4 / 64 + 2;

struct Shared {
  union {
    uint64_t list[kList];
    uint64_t seg[kSegs];
  };
  uint64_t hist[kBins];
  uint64_t red[16];
  uint64_t val[2];
  int32_t n;
};

__device__ inline uint64_t pair_of(uint32_t key, int32_t id) {
  return uint64_t(key) << 32 | uint32_t(~id);
}
__device__ inline uint32_t key_in(uint64_t pair) { return uint32_t(pair >> 32); }
__device__ inline int32_t id_in(uint64_t pair) { return int32_t(~uint32_t(pair)); }

// Appends to the list the tokens that `take` accepts; false when they are more than kList.
template <int DT, class F>
__device__ bool collect(const Row<DT> &row, Shared &sh, F take) {
  const int lane = threadIdx.x & 63;
  __syncthreads();
  if (threadIdx.x == 0) sh.n = 0;
  __syncthreads();
  const int32_t rounds = (row.groups() + kThreads - 1) / kThreads;
  for (int32_t r = 0; r < rounds; ++r) {
    const int32_t g = r * kThreads + threadIdx.x;
    uint64_t got[8];
    int n = 0;
    row.visit(g, [&](int32_t id, float x) {
      const uint32_t key = key_of(x);
      if (take(key)) {
        // n is at most kVec: the unrolled choice keeps got[] in registers
#pragma unroll
        for (int e = 0; e < 8; ++e) got[e] = e == n ? pair_of(key, id) : got[e];
        ++n;
      }
    });
    if (__any(n > 0)) {
      int x = n;
      for (int w = 1; w < 64; w <<= 1) {
        const int y = __shfl_up(x, w, 64);
        if (lane >= w) x += y;
      }
      int base = 0;
      if (lane == 63) base = atomicAdd(&sh.n, x);
      base = __shfl(base, 63, 64) + x - n;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n && base + e < kList) sh.list[base + e] = got[e];
    }
  }
  __syncthreads();
  return sh.n <= kList;
}

// Fills the list up to a power of two and sorts it; returns its length.
__device__ int sort_list(Shared &sh) {
  const int n = sh.n;
  int n2 = 64;
  while (n2 < n) n2 <<= 1;
  for (int i = n + threadIdx.x; i < n2; i += kThreads) sh.list[i] = 0;
  __syncthreads();
  sort_down(sh.list, n2);
  return n;
}

template <int DT>
__device__ void sample_slow(const SampleArgs &a, const char *base, int32_t row, const Weigh &weigh,
                            float tp, uint64_t least, int32_t k_in, float u, Shared &sh);

template <int DT>
__global__ void __launch_bounds__(kThreads) k_sample(SampleArgs a) {
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t row = blockIdx.x, V = a.vocab;
  const char *base = static_cast<const char *>(a.logits) +
                     int64_t(row) * a.stride * (DT == FS_F32 ? 4 : 2);
  const Row<DT> r(base, V);
  const float T = a.temperature ? a.temperature[row] : 1.f;
  const float tp = a.top_p ? a.top_p[row] : 1.f, mp = a.min_p ? a.min_p[row] : 0.f;
  const float u = a.u[row];
  const int32_t k_in = a.top_k ? a.top_k[row] : 0;
  const bool bad = !(T >= 0.f) || !(T < INFINITY) || !(tp >= 0.f && tp <= 1.f) ||
                   !(mp >= 0.f && mp <= 1.f) || !(u >= 0.f && u < 1.f);

  // the largest logit and its lowest id
  uint64_t mine = 0;
  for (int32_t g = tid; g < r.groups(); g += kThreads)
    r.visit(g, [&](int32_t id, float x) {
      const uint64_t c = pair_of(key_of(x), id);
      mine = c > mine ? c : mine;
    });
  uint64_t best = mine;
  for (int w = 32; w; w >>= 1) {
    const uint64_t o = __shfl_xor(best, w, 64);
    best = o > best ? o : best;
  }
  if (lane == 0) sh.red[wave] = best;
  __syncthreads();
  for (int i = 0; i < kThreads / 64; ++i) best = sh.red[i] > best ? sh.red[i] : best;
  const uint32_t top = key_in(best);
  if (bad || top <= kLow || T == 0.f) {
    if (tid == 0) {
      const bool none = bad || top <= kLow;
      a.token[row] = none ? -1 : id_in(best);
      if (a.logprob) a.logprob[row] = none ? -INFINITY : 0.f;
      if (a.kept) a.kept[row] = none ? 0 : 1;
      if (bad) raise_err(a.err, FS_E_RANGE);
    }
    return;
  }
  const Weigh weigh{top, double(value_of(top)), 1.4426950408889634 / double(T)};
  uint64_t least = uint64_t(ceil(__dmul_rn(double(mp), kOne)));
  if (least < 1) least = 1;

  // kept: pairs (key, ~id) of at least `cut`, with a weight of at least `least`
  uint64_t cut = uint64_t(kLow + 1) << 32;
  if (k_in > 0 && k_in < V) {
    // The k-th largest of the threads' own largest keys is no larger than the k-th
    // largest key: what is at least that holds the first k tokens.
    if (k_in > kThreads)
      return sample_slow<DT>(a, base, row, weigh, tp, least, k_in, u, sh);
    __syncthreads();
    sh.list[tid] = mine;
    __syncthreads();
    sort_down(sh.list, kThreads);
    const uint32_t bound = max(key_in(sh.list[k_in - 1]), kLow + 1);
    if (!collect<DT>(r, sh, [&](uint32_t key) { return key >= bound; }))
      return sample_slow<DT>(a, base, row, weigh, tp, least, k_in, u, sh);
    const int n = sort_list(sh);
    // the list's order is the definition's: every cut is a prefix of it
    const int per = (n + kThreads - 1) / kThreads, i0 = min(tid * per, n), i1 = min(i0 + per, n);
    uint64_t w[kList / kThreads], sum = 0;
#pragma unroll
    for (int e = 0; e < kList / kThreads; ++e) {
      const int i = i0 + e;
      w[e] = i < i1 && i < k_in ? weigh(key_in(sh.list[i])) : 0;
      sum += w[e];
    }
    uint64_t before = block_scan(sum, sh.red);
    const uint64_t W = block_sum(sum, sh.red);
    uint64_t limit = ~uint64_t(0);
    if (tp < 1.f) {
      const double lim = ceil(__dmul_rn(double(tp), double(W)));
      limit = lim < 1.0 ? 1 : uint64_t(lim);
    }
    uint64_t kept = 0, kept_n = 0;
#pragma unroll
    for (int e = 0; e < kList / kThreads; ++e) {
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
    // the kept ones by id, with their weights: ids sort upward as ~id downward
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kList / kThreads; ++e) {
      const int i = i0 + e;
      if (i < i1 && w[e]) sh.list[i] = uint64_t(uint32_t(sh.list[i])) << 32 | key_in(sh.list[i]);
    }
    __syncthreads();
    if (tid == 0) sh.n = m;
    __syncthreads();
    sort_list(sh);
    const int per2 = (m + kThreads - 1) / kThreads, j0 = min(tid * per2, m),
              j1 = min(j0 + per2, m);
    sum = 0;
#pragma unroll
    for (int e = 0; e < kList / kThreads; ++e) {
      w[e] = j0 + e < j1 ? weigh(uint32_t(sh.list[j0 + e])) : 0;
      sum += w[e];
    }
    uint64_t run = block_scan(sum, sh.red);
    if (run <= goal && goal < run + sum) {
      bool found = false;
#pragma unroll
      for (int e = 0; e < kList / kThreads; ++e) {
        run += w[e];
        if (!found && w[e] && run > goal) {
          found = true;
          a.token[row] = int32_t(~key_in(sh.list[j0 + e]));
          if (a.logprob) a.logprob[row] = float(log(double(w[e]) / double(S)));
          if (a.kept) a.kept[row] = m;
        }
      }
    }
    return;
  }

  if (tp < 1.f) {
    // weights by bin of y, 32 bins to an octave
    for (int i = tid; i < kBins; i += kThreads) sh.hist[i] = 0;
    __syncthreads();
    for (int32_t g = tid; g < r.groups(); g += kThreads)
      r.visit(g, [&](int32_t, float x) {
        const double y = weigh.y_of(key_of(x));
        const uint64_t w = weight_of(y);
        if (w)
          atomicAdd(reinterpret_cast<unsigned long long *>(&sh.hist[int(y * 32.0)]),
                    (unsigned long long)w);
      });
    __syncthreads();
    // the bin in which the running sum reaches the limit
    constexpr int kPer = (kBins + kThreads - 1) / kThreads;
    uint64_t h[kPer], sum = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      h[e] = tid * kPer + e < kBins ? sh.hist[tid * kPer + e] : 0;
      sum += h[e];
    }
    uint64_t before = block_scan(sum, sh.red);
    const uint64_t W = block_sum(sum, sh.red);
    const double lim = ceil(__dmul_rn(double(tp), double(W)));
    const uint64_t limit = lim < 1.0 ? 1 : uint64_t(lim);
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      if (before < limit && before + h[e] >= limit) {
        sh.val[0] = before;
        sh.val[1] = tid * kPer + e;
      }
      before += h[e];
    }
    __syncthreads();
    const uint64_t above = sh.val[0];
    const int bin = int(sh.val[1]);
    if (!collect<DT>(r, sh, [&](uint32_t key) {
          if (key <= kLow) return false;
          const double y = weigh.y_of(key);
          return y < 41.0 && int(y * 32.0) == bin;
        }))
      return sample_slow<DT>(a, base, row, weigh, tp, least, k_in, u, sh);
    const int n = sort_list(sh);
    const int per = (n + kThreads - 1) / kThreads, i0 = min(tid * per, n), i1 = min(i0 + per, n);
    uint64_t w[kList / kThreads];
    sum = 0;
#pragma unroll
    for (int e = 0; e < kList / kThreads; ++e) {
      w[e] = i0 + e < i1 ? weigh(key_in(sh.list[i0 + e])) : 0;
      sum += w[e];
    }
    before = above + block_scan(sum, sh.red);
    // the last token whose predecessors stay below the limit
#pragma unroll
    for (int e = 0; e < kList / kThreads; ++e) {
      if (w[e] && before < limit && before + w[e] >= limit) sh.val[0] = sh.list[i0 + e];
      before += w[e];
    }
    __syncthreads();
    cut = sh.val[0];
  }

  // the kept weights in the order of ids: a sum for each 64 groups, then the one that
  // holds the goal, token by token
  __syncthreads();
  const int32_t segs = (r.groups() + 63) / 64;
  uint64_t total = 0;
  uint32_t count = 0;
  auto kept_weight = [&](int32_t id, float x) -> uint64_t {
    const uint32_t key = key_of(x);
    if (pair_of(key, id) < cut) return 0;
    const uint64_t w = weigh(key);
    return w >= least ? w : 0;
  };
  for (int32_t s = wave; s < segs; s += kThreads / 64) {
    uint64_t sum = 0;
    r.visit(s * 64 + lane, [&](int32_t id, float x) {
      const uint64_t w = kept_weight(id, x);
      sum += w;
      count += w != 0;
    });
    for (int w = 32; w; w >>= 1) sum += __shfl_xor(sum, w, 64);
    if (lane == 0) sh.seg[s] = sum;
    total += sum;
  }
  const uint64_t S = block_sum(lane == 0 ? total : uint64_t(0), sh.red);
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
  sum = 0;
  r.visit(g, [&](int32_t id, float x) { sum += kept_weight(id, x); });
  uint64_t x = sum;
  for (int w = 1; w < 64; w <<= 1) {
    const uint64_t y = __shfl_up(x, w, 64);
    if (lane >= w) x += y;
  }
  run += x - sum;
  if (run <= goal && goal < run + sum) {
    bool found = false;
    r.visit(g, [&](int32_t id, float v) {
      const uint64_t w = kept_weight(id, v);
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
template <int DT>
__device__ __noinline__ void sample_slow(const SampleArgs &a, const char *base, int32_t row,
                                         const Weigh &weigh, float tp, uint64_t least,
                                         int32_t k_in, float u, Shared &sh) {
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
          if (w) atomicAdd(reinterpret_cast<unsigned long long *>(&hist[(key >> shift) & 255]), w);
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

}  // namespace

size_t sample_workspace_bytes(int32_t, int32_t, int32_t) { return 0; }

hipError_t launch_sample(int32_t dtype, int32_t rows, int32_t vocab, const void *logits,
                         int64_t stride, const fs_sampling *p, const float *u, int32_t *token,
                         float *logprob, int32_t *kept, void *ws, int32_t *err,
                         hipStream_t stream) {
  SampleArgs a{logits, stride,   rows, vocab, p->temperature, p->top_p, p->min_p, u, p->top_k,
               token,  kept,     logprob, err};
  const dim3 grid(rows), block(kThreads);
  if (dtype == FS_BF16)
    hipLaunchKernelGGL(k_sample<FS_BF16>, grid, block, 0, stream, a);
  else if (dtype == FS_F16)
    hipLaunchKernelGGL(k_sample<FS_F16>, grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL(k_sample<FS_F32>, grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace fs
