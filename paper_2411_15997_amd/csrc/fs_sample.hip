// The next token of each row from its logits and one given random number, in whole-number
// weights (2^40 for the largest logit): every sum is exact, so the kept set and the token
// do not depend on the order of additions.  One work-group per row; the cuts of top-k and
// top-p are found digit by digit of an order-preserving 32-bit key of the logit.
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
__device__ inline float load_logit(const void *row, int32_t i) {
  if constexpr (DT == FS_F32)
    return static_cast<const float *>(row)[i];
  else
    return to_f32<DT == FS_BF16>(static_cast<const short *>(row)[i]);
}

// 2^-y for y >= 0 times 2^40, rounded down.  2^f for |f| <= 1/2 by the Taylor series of
// exp(f ln 2) (degree 12: below 2e-16 of the value).
__device__ inline uint64_t weight_of(double y) {
  if (!(y < 41.0)) return 0;
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
  return uint64_t(ldexp(p, int(k) + 40));
}

struct Weigh {
  uint32_t top;  // key of the largest logit
  double best, per;
  __device__ uint64_t operator()(uint32_t key) const {
    if (key == top) return uint64_t(1) << 40;
    return weight_of(__dmul_rn(__dsub_rn(best, double(value_of(key))), per));
  }
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

template <int DT>
__global__ void __launch_bounds__(kThreads) k_sample(SampleArgs a) {
  __shared__ uint64_t red[16];
  __shared__ uint64_t hist[256];
  __shared__ uint64_t sh_u64;
  __shared__ uint32_t sh_key;
  __shared__ int32_t sh_id;
  const int tid = threadIdx.x;
  const int32_t row = blockIdx.x, V = a.vocab;
  const char *base = static_cast<const char *>(a.logits) +
                     int64_t(row) * a.stride * (DT == FS_F32 ? 4 : 2);
  const float T = a.temperature ? a.temperature[row] : 1.f;
  const float tp = a.top_p ? a.top_p[row] : 1.f, mp = a.min_p ? a.min_p[row] : 0.f;
  const float u = a.u[row];
  const int32_t k_in = a.top_k ? a.top_k[row] : 0;
  const bool bad = !(T >= 0.f) || !(T < INFINITY) || !(tp >= 0.f && tp <= 1.f) ||
                   !(mp >= 0.f && mp <= 1.f) || !(u >= 0.f && u < 1.f);

  // the largest logit and its lowest id
  uint64_t best = 0;
  for (int32_t i = tid; i < V; i += kThreads) {
    const uint64_t c = uint64_t(key_of(load_logit<DT>(base, i))) << 32 | uint32_t(~i);
    best = c > best ? c : best;
  }
  for (int w = 32; w; w >>= 1) {
    const uint64_t o = __shfl_xor(best, w, 64);
    best = o > best ? o : best;
  }
  if ((tid & 63) == 0) red[tid >> 6] = best;
  __syncthreads();
  for (int i = 0; i < kThreads / 64; ++i) best = red[i] > best ? red[i] : best;
  const uint32_t top = uint32_t(best >> 32);
  if (bad || top <= kLow || T == 0.f) {
    if (tid == 0) {
      const bool none = bad || top <= kLow;
      a.token[row] = none ? -1 : int32_t(~uint32_t(best));
      if (a.logprob) a.logprob[row] = none ? -INFINITY : 0.f;
      if (a.kept) a.kept[row] = none ? 0 : 1;
      if (bad) raise_err(a.err, FS_E_RANGE);
    }
    return;
  }
  Weigh weigh{top, double(value_of(top)), 1.4426950408889634 / double(T)};

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
      prefix = sh_key;
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
      prefix = sh_key;
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
  uint64_t least = uint64_t(ceil(__dmul_rn(double(mp), kOne)));
  if (least < 1) least = 1;

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
