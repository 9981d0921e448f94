// A projection with every request's own low-rank adapter beside the shared weight:
//   y = x W^T + scale_a (x A_a^T) B_a^T,   a = the row's request's adapter.
// Two launches: k_shrink makes h = scale x A_a^T per request in fp32 and stores it as the
// sum of two 16-bit values; k_linear runs the product over K and then goes on over the
// few columns of h against B_a in the same accumulators, so y is written once and never
// read.
#include "fs_engine.h"

namespace fs {

namespace {

struct LinArgs {
  const int32_t *q_off, *adapter, *rank;
  const float *scale;
  int32_t n_seqs, rows, K, N, n_adapters, R;  // R: max_rank (0: no adapters)
  const short *x, *w, *a, *b;
  short *y;
  short *h;  // [rows][2R]: high parts, low parts
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

// One request's rows, 16 at a time, against 16 of its adapter's A rows; the four waves
// share out K and join in LDS.
template <bool BF>
__global__ void __launch_bounds__(256) k_shrink(LinArgs g) {
  __shared__ float part[4][16][17];
  const RowTile t = row_tile<4>(g.q_off, g.n_seqs, blockIdx.x);
  if (t.rows <= 0) return;
  int32_t code = 0, rank;
  const int32_t ad = adapter_of(g, t.s, rank, code);
  if (threadIdx.x == 0 && blockIdx.y == 0) raise_err(g.err, code);
  const int j0 = blockIdx.y * 16;
  if (ad < 0) return;  // k_linear does not look at h for such rows
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, kq = (lane >> 4) * 8;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  if (j0 < rank) {
    const short *xp = g.x + int64_t(t.row0 + min(r, t.rows - 1)) * g.x_stride;
    const short *ap = g.a + (int64_t(ad) * g.R + min(j0 + r, rank - 1)) * g.K;
    const s16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int k = wave * 32 + kq; k < (g.K + 31) / 32 * 32; k += 128) {
      const s16x8 xv = k < g.K ? *reinterpret_cast<const s16x8 *>(xp + k) : zero;
      const s16x8 av = k < g.K ? *reinterpret_cast<const s16x8 *>(ap + k) : zero;
      acc = mfma_16x16x32<BF>(xv, av, acc);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) part[wave][(lane >> 4) * 4 + i][r] = acc[i];
  __syncthreads();
  const int row = threadIdx.x >> 4, j = threadIdx.x & 15;
  if (row < t.rows && j0 + j < g.R) {
    float v = (part[0][row][j] + part[1][row][j]) + (part[2][row][j] + part[3][row][j]);
    v = j0 + j < rank ? v * (g.scale ? __ldg(g.scale + ad) : 1.f) : 0.f;
    const short hi = to_16<BF>(v);
    short *hp = g.h + int64_t(t.row0 + row) * (2 * g.R) + j0 + j;
    hp[0] = hi;
    hp[g.R] = to_16<BF>(v - to_f32<BF>(hi));
  }
}

// One wave: 16 rows by 64 columns, operands straight from memory in the matrix cores'
// layout.
template <bool BF>
__global__ void __launch_bounds__(256) k_linear(LinArgs g) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, kq = (lane >> 4) * 8;
  const int n0 = (blockIdx.x * 4 + wave) * 64, m0 = blockIdx.y * 16;
  if (n0 >= g.N) return;
  const int row = min(m0 + r, g.rows - 1);
  const s16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
  f32x4 acc[4] = {};
  const short *xp = g.x + int64_t(row) * g.x_stride;
  const short *wp[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) wp[c] = g.w + int64_t(min(n0 + 16 * c + r, g.N - 1)) * g.K;
  for (int k = kq; k < (g.K + 31) / 32 * 32; k += 32) {
    const s16x8 xv = k < g.K ? *reinterpret_cast<const s16x8 *>(xp + k) : zero;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const s16x8 wv = k < g.K ? *reinterpret_cast<const s16x8 *>(wp[c] + k) : zero;
      acc[c] = mfma_16x16x32<BF>(xv, wv, acc[c]);
    }
  }
  if (g.n_adapters > 0) {
    const int last = min(m0 + 15, g.rows - 1);
    for (int s = seq_of_row(g.q_off, g.n_seqs, m0); s < g.n_seqs && __ldg(g.q_off + s) <= last;
         ++s) {
      int32_t code = 0, rank;
      const int32_t ad = adapter_of(g, s, rank, code);
      if (ad < 0 || rank == 0) continue;
      const bool mine = m0 + r >= __ldg(g.q_off + s) && m0 + r < __ldg(g.q_off + s + 1);
      const short *hp = g.h + int64_t(row) * (2 * g.R);
      // chunks of 8 columns: R/8 high ones, then R/8 low ones
      for (int c8 = lane >> 4; c8 < (g.R / 4 + 3) / 4 * 4; c8 += 4) {
        const bool in = c8 < g.R / 4;
        const s16x8 hv = mine && in ? *reinterpret_cast<const s16x8 *>(hp + c8 * 8) : zero;
        const int j = (c8 < g.R / 8 ? c8 : c8 - g.R / 8) * 8;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          s16x8 bv = zero;
          if (in && j < rank) {
            bv = *reinterpret_cast<const s16x8 *>(
                g.b + (int64_t(ad) * g.N + min(n0 + 16 * c + r, g.N - 1)) * g.R + j);
#pragma unroll
            for (int i = 0; i < 8; ++i) bv[i] = j + i < rank ? bv[i] : short(0);
          }
          acc[c] = mfma_16x16x32<BF>(hv, bv, acc[c]);
        }
      }
    }
  }
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int m = m0 + (lane >> 4) * 4 + i, n = n0 + 16 * c + r;
      if (m < g.rows && n < g.N) g.y[int64_t(m) * g.y_stride + n] = to_16<BF>(acc[c][i]);
    }
}

template <bool BF>
void run(const LinArgs &g, int64_t tiles, hipStream_t stream) {
  if (g.n_adapters > 0)
    hipLaunchKernelGGL(k_shrink<BF>, dim3(tiles, (g.R + 15) / 16), dim3(256), 0, stream, g);
  hipLaunchKernelGGL(k_linear<BF>, dim3((g.N + 255) / 256, (g.rows + 15) / 16), dim3(256), 0,
                     stream, g);
}

}  // namespace

size_t adapter_workspace_bytes(const fs_step *s, const fs_adapters *ad) {
  if (ad->n_adapters == 0) return 0;
  return size_t(s->q_off_h[s->n_seqs]) * ad->max_rank * 4;
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
  g.x_stride = x_stride;
  g.y_stride = y_stride;
  g.err = err;
  const int64_t tiles = row_tiles(s, 4);
  if (ad->dtype == FS_BF16)
    run<true>(g, tiles, stream);
  else
    run<false>(g, tiles, stream);
  return hipGetLastError();
}

}  // namespace fs
