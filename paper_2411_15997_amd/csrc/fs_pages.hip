// The pages of a cache: letting rows go, forking rows that share a prompt's pages, moving the
// pages in use together, and copying pages.
//
// A page's state is its count of holders.  Free pages are taken, and pages are moved, in the
// order of ids: a page's place is its rank among its kind, the sum of a block's count before it
// (k_pages_count, then each block adds up the counts of those before it) and of ballots inside the
// block.  So no result hangs on the order of atomics; those used (claims by the lowest index,
// counts of holders) end the same in any order.
// Bound by launches and chains of a few dependent loads: pools of up to 2,048 pages take one kernel
// of 4 to 8 us, larger ones three of 3 to 6 (256 forks among 9,425 pages 13 us, 9,559 pages moved
// together 15); the copies by their bytes (277 MB: 46 us, 6.0 TB/s, some of it from the cache before
// memory).
#include "fs_cache.h"

namespace fs {

namespace {

constexpr int kBlock = 1024;          // threads
constexpr int kPer = 2 * kBlock;      // pages of a work-group
constexpr int kFewPages = 2 * kBlock;  // a pool that one work-group looks through
constexpr int kFewForks = 32;         // forks, and rows, that the same one finishes
constexpr int kSomeForks = 256;       // forks that it plans
constexpr int kClaims = 8192;         // rows whose claims LDS holds

struct PoolArgs {
  int32_t n_pages, page_shift, n_rows, width;
  int32_t *refs, *table, *held;
  int64_t stride;
  int32_t n, blocks;
  const int32_t *rows, *parent, *child, *shared, *room;
  int32_t *src, *dst, *count, *refs_out, *table_out;
  int64_t out_stride;
  int32_t *claim;            // [n_rows]
  int32_t *first;            // [n]: new pages of the forks before; -1 - that for a refused one
  int32_t *block_sum;        // [blocks]
  int32_t *list;             // [n_pages]: free pages in order; of a compaction: which moved page it
                             // is, 0 for one that stays, -1 for a free one
  int32_t most;              // free pages that a fork can take
  int32_t *word;             // fork: whether the pages suffice; compaction: L and the moves
  int32_t *err;
};

// Sum over the work-group of x, in every thread.
template <class T>
__device__ inline T block_total(T x, T *lds) {
#pragma unroll
  for (int w = 32; w; w >>= 1) x += __shfl_xor(x, w, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  T sum = 0;
#pragma unroll
  for (int i = 0; i < kBlock / 64; ++i) sum += lds[i];
  return sum;
}
// The sum of x over the threads before this one.
template <class T>
__device__ inline T block_before(T x, T *lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T run = x;
#pragma unroll
  for (int w = 1; w < 64; w <<= 1) {
    const T y = __shfl_up(run, w, 64);
    if (lane >= w) run += y;
  }
  __syncthreads();
  if (lane == 63) lds[wave] = run;
  __syncthreads();
  T before = run - x;
  for (int i = 0; i < wave; ++i) before += lds[i];
  return before;
}

// Whether fork i (parent p, sh shared tokens) would share a page id out of range, or a free page
// (which another one may get as a new one): first[i] is then -1, else 0.  Seen before the plan: a
// refused fork takes no free pages from the others.  By `lanes` neighbouring lanes (a power of two up
// to 64) of threads that all come here.
__device__ inline void check_shared(const PoolArgs &a, int32_t i, int32_t p, int32_t sh, int lanes) {
  const int lane = threadIdx.x & (lanes - 1);
  const bool any = i < a.n && p >= 0 && p < a.n_rows && sh > 0;
  // (what the parent does not hold is refused for that)
  const int32_t pages =
      any ? int32_t(min((int64_t(sh) + (1 << a.page_shift) - 1) >> a.page_shift, int64_t(a.width)))
          : 0;
  const int32_t *from = a.table + int64_t(any ? p : 0) * a.stride;
  int32_t bad = 0;
  for (int32_t j = lane; j < pages; j += lanes) {
    const uint32_t id = from[j];
    bad |= id >= uint32_t(a.n_pages) || a.refs[id] <= 0;
  }
  for (int w = lanes >> 1; w; w >>= 1) bad |= __shfl_xor(bad, w, 64);
  if (lane == 0 && i < a.n) a.first[i] = -bad;
}

// Which forks are sound (first[i] says which share sound pages) and how many new pages come before
// each one's, by one work-group; the sum, at most n_pages + 1.
__device__ inline int32_t plan_forks(const PoolArgs &a) {
  __shared__ int64_t lds64[kBlock / 64];
  __shared__ int32_t lds_claim[kClaims];
  const int tid = threadIdx.x;
  // A child belongs to the lowest index that names it.  (Atomics alone, in LDS where that holds
  // the rows: no other work-group looks at the claims, so nothing has to be flushed.)
  int32_t *const claim = a.n_rows <= kClaims ? lds_claim : a.claim;
  for (int32_t i = tid; i < a.n; i += kBlock)
    if (uint32_t(a.child[i]) < uint32_t(a.n_rows)) atomicExch(claim + a.child[i], INT32_MAX);
  __syncthreads();
  for (int32_t i = tid; i < a.n; i += kBlock)
    if (uint32_t(a.child[i]) < uint32_t(a.n_rows)) atomicMin(claim + a.child[i], i);
  __syncthreads();
  const int64_t most = int64_t(a.n_pages) + 1;  // more than there are is as many as that
  int64_t before = 0;
  for (int32_t i0 = 0; i0 < a.n; i0 += kBlock) {
    const int32_t i = i0 + tid;
    int64_t need = 0;
    bool ok = false;
    if (i < a.n) {
      const int32_t p = a.parent[i], c = a.child[i], sh = a.shared[i], room = a.room[i];
      const int32_t size = 1 << a.page_shift;
      ok = p >= -1 && p < a.n_rows && uint32_t(c) < uint32_t(a.n_rows) && sh >= 0 && room >= sh;
      const int32_t has = ok && p >= 0 ? a.held[p] : 0, own = ok ? a.held[c] : 0;
      if (ok) ok = atomicMin(claim + c, INT32_MAX) == i && own == 0;
      const int32_t pages = int32_t((int64_t(room) + size - 1) >> a.page_shift);
      if (ok) ok = pages <= a.width;
      if (ok && sh > 0)
        ok = p >= 0 && has >= 0 && has <= a.width &&
             int32_t((int64_t(sh) + size - 1) >> a.page_shift) <= has && a.first[i] == 0;
      if (ok)
        need = pages - (sh >> a.page_shift);
      else
        raise_err(a.err, FS_E_RANGE);
    }
    const int64_t f = min(before + block_before(need, lds64), most);
    before += block_total(need, lds64);
    if (i < a.n) a.first[i] = int32_t(ok ? f : -1 - f);
  }
  return int32_t(min(before, most));
}
__device__ inline bool enough(const PoolArgs &a, int32_t wanted, int32_t free) {
  if (threadIdx.x == 0) {
    *a.word = wanted <= free;  // (read by k_pages_fork)
    if (wanted > free) raise_err(a.err, FS_E_OVERFLOW);
  }
  return wanted <= free;
}

// Fork i by THREADS threads (a wave, or a work-group): the child's row, counts and the page to be
// copied.
template <int THREADS>
__device__ inline void fork_row(const PoolArgs &a, int32_t i) {
  const int tid = threadIdx.x % THREADS;
  const int32_t first = a.first[i];
  const bool go = first >= 0 && *a.word;
  const int32_t p = go ? a.parent[i] : 0, c = go ? a.child[i] : 0, sh = go ? a.shared[i] : 0;
  const int32_t size = 1 << a.page_shift, full = sh >> a.page_shift;
  const int32_t pages = go ? int32_t((int64_t(a.room[i]) + size - 1) >> a.page_shift) : 0;
  const bool part = sh & (size - 1);
  const int32_t *from = a.table + int64_t(max(p, 0)) * a.stride;  // (ids looked at before the plan)
  if (tid == 0) {
    a.src[i] = go && part ? from[full] : -1;
    a.dst[i] = go && part ? a.list[first] : -1;
    if (go) a.held[c] = pages;
  }
  if (!go) return;
  int32_t *to = a.table + int64_t(c) * a.stride;
  for (int32_t j = tid; j < pages; j += THREADS) {
    const int32_t id = j < full ? from[j] : a.list[first + j - full];
    to[j] = id;
    atomicAdd(a.refs + id, 1);
  }
}

// Pools of few pages, by one work-group: a wave goes through its share of the ids 64 at a time.
// f(p, refs) of the share's pages (refs 0 past the last).
template <class F>
__device__ inline void my_pages(const PoolArgs &a, F f) {
  const int32_t share = (a.n_pages + kBlock - 1) / kBlock * 64;  // of a wave
  const int32_t from = int32_t(threadIdx.x >> 6) * share, to = min(from + share, a.n_pages);
  for (int32_t p0 = from; p0 < to; p0 += 64 * 8) {  // eight loads under way
    const int32_t p = p0 + int32_t(threadIdx.x & 63);
    int32_t refs[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) refs[i] = p + 64 * i < a.n_pages ? a.refs[p + 64 * i] : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (p0 + 64 * i < to) f(p + 64 * i, refs[i]);
  }
}
__device__ inline int32_t lanes_before(uint64_t lanes) {
  return __popcll(lanes & ((uint64_t(1) << (threadIdx.x & 63)) - 1));
}
// The sum over the waves before this one of x (one for all lanes of a wave), and over all.
__device__ inline int32_t waves_before(int32_t x, int32_t *lds, int32_t &all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
  if (lane == 0) lds[wave] = x;
  __syncthreads();
  int32_t before = 0;
  all = 0;
#pragma unroll
  for (int i = 0; i < kBlock / 64; ++i) {
    if (i < wave) before += lds[i];
    all += lds[i];
  }
  return before;
}

// The forks, and the list of the first free pages, as many as they take, in order of ids.  WHOLE:
// the rows of few forks too, two for each wave.  (Eight forks in a pool of 247 pages: 8.1 us, 11.3
// and two more launches with the kernels for many.  256 forks that share 7 pages each in a pool of
// 2,000: 12.4 with k_pages_fork, 13.1 and one more launch; 1,024 that share 75: 35.3 and 19.8.)
template <bool WHOLE>
__global__ void __launch_bounds__(kBlock) k_pages_plan(PoolArgs a) {
  __shared__ int32_t lds[kBlock / 64];
  int32_t mine = 0, all;
  // this thread's fork to be checked (2^shift lanes for each), its loads under way with the pages'
  const int shift = min(6, __clz(a.n - 1) - (32 - 10));
  const int32_t i = int32_t(threadIdx.x) >> shift;
  const int32_t parent = i < a.n ? a.parent[i] : -1, shared = i < a.n ? a.shared[i] : 0;
  my_pages(a, [&](int32_t p, int32_t refs) {
    mine += __popcll(__ballot(p < a.n_pages && refs <= 0));
  });
  check_shared(a, i, parent, shared, 1 << shift);
  const int32_t wanted = plan_forks(a);
  int32_t at = waves_before(mine, lds, all);
  if (enough(a, wanted, all))
    my_pages(a, [&](int32_t p, int32_t refs) {
      const uint64_t free = __ballot(p < a.n_pages && refs <= 0);
      const int32_t to = at + lanes_before(free);
      if (p < a.n_pages && refs <= 0 && to < wanted) a.list[to] = p;
      at += __popcll(free);
    });
  if constexpr (WHOLE) {
    __syncthreads();  // what the waves have written is read by others of this work-group
    for (int32_t i = threadIdx.x >> 6; i < a.n; i += kBlock / 64) fork_row<64>(a, i);
  }
}

// Pools of many pages: the pages of block b that are in use (LIVE) or free, and for a fork, in
// blocks of their own, the shared pages of a fork for each wave.
template <bool LIVE>
__global__ void __launch_bounds__(kBlock) k_pages_count(PoolArgs a) {
  __shared__ int32_t lds[kBlock / 64];
  const int tid = threadIdx.x, b = blockIdx.x;
  if (LIVE || b < a.blocks) {
    int32_t x = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int32_t p = b * kPer + i * kBlock + tid;
      if (p < a.n_pages) x += (a.refs[p] > 0) == LIVE;
    }
    x = block_total(x, lds);
    if (tid == 0) a.block_sum[b] = x;
  } else {
    const int32_t i = (b - a.blocks) * (kBlock / 64) + (tid >> 6);
    check_shared(a, i, i < a.n ? a.parent[i] : -1, i < a.n ? a.shared[i] : 0, 64);
  }
}

// The list of the first free pages, as many as can be asked for, and, in a block of its own, the
// forks.
__global__ void __launch_bounds__(kBlock) k_pages_list(PoolArgs a) {
  __shared__ int32_t lds[kBlock / 64];
  const int tid = threadIdx.x;
  const bool plans = int32_t(blockIdx.x) == a.blocks;
  int32_t before = 0;  // free pages of the blocks before: for the forks, all
  for (int32_t b = tid; b < int32_t(blockIdx.x); b += kBlock) before += a.block_sum[b];
  before = block_total(before, lds);
  if (plans) {
    enough(a, plan_forks(a), before);
    return;
  }
  if (before >= a.most) return;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int32_t p = blockIdx.x * kPer + i * kBlock + tid;
    const int32_t is = p < a.n_pages && a.refs[p] <= 0;
    const int32_t at = before + block_before(is, lds);
    if (is && at < a.most) a.list[at] = p;
    before += block_total(is, lds);
  }
}

__global__ void __launch_bounds__(256) k_pages_fork(PoolArgs a) { fork_row<256>(a, blockIdx.x); }

// Row r let go, by the work-group.
__device__ inline void free_row(const PoolArgs &a, int32_t r, int32_t &got) {
  const int tid = threadIdx.x;
  if (uint32_t(r) >= uint32_t(a.n_rows)) {
    if (tid == 0) raise_err(a.err, FS_E_RANGE);
    return;
  }
  if (tid == 0) got = atomicExch(a.held + r, 0);  // of a row named twice, one gets them
  __syncthreads();
  int32_t n = got;
  bool bad = n < 0 || n > a.width;
  if (bad) n = 0;
  const int32_t *row = a.table + int64_t(r) * a.stride;
  for (int32_t j = tid; j < n; j += 256) {
    const int32_t id = row[j];
    if (uint32_t(id) >= uint32_t(a.n_pages)) {
      bad = true;
    } else if (atomicSub(a.refs + id, 1) <= 0) {
      atomicAdd(a.refs + id, 1);
      bad = true;
    }
  }
  if (bad) raise_err(a.err, FS_E_RANGE);
}

// (A launch counts its threads in 32 bits: 2^24 work-groups would be none.)
constexpr int kFreeBlocks = 65536;
__global__ void __launch_bounds__(256) k_pages_free(PoolArgs a) {
  __shared__ int32_t got;
  free_row(a, a.rows[blockIdx.x], got);
  for (uint32_t i = blockIdx.x + kFreeBlocks; i < uint32_t(a.n); i += kFreeBlocks) {
    __syncthreads();  // (got was the last row's)
    free_row(a, a.rows[i], got);
  }
}

// Page p of a compaction, `rank` pages in use before it, L in all and `below` of them below L: the
// pages in use with ids from L on, and the free ones below, in order of ids are src and dst.
__device__ inline void place_page(const PoolArgs &a, int32_t p, int32_t refs, int32_t rank, int32_t L,
                                  int32_t below) {
  const int32_t moves = L - below;
  a.list[p] = refs <= 0 ? -1 : p < L ? 0 : rank - below;
  if (p < L && refs <= 0) a.dst[p - rank] = p;
  if (p >= L && refs > 0) a.src[rank - below] = p;
  if (a.refs_out != a.refs) a.refs_out[p] = p < L && refs > 0 ? refs : 0;
  if (p >= moves && p < a.n_pages / 2) a.src[p] = a.dst[p] = -1;
}
__device__ inline void put_moves(const PoolArgs &a, int32_t L, int32_t below) {
  *a.count = L - below;
  a.word[0] = L;
  a.word[1] = L - below;
}

// Counts of the moved pages `from`, `from` + step .. .
__device__ inline void move_counts(const PoolArgs &a, int32_t moves, int32_t from, int32_t step) {
  for (int32_t i = from; i < moves; i += step) {
    const int32_t s = a.src[i], d = a.dst[i];
    const int32_t x = a.refs[s];
    a.refs_out[s] = 0;
    a.refs_out[d] = x;
  }
}
// The ids of row r, entries `from`, `from` + step .. .
__device__ inline void remap_row(const PoolArgs &a, int32_t L, int32_t r, int32_t from,
                                 int32_t step) {
  int32_t held = a.held[r];
  bool bad = held < 0 || held > a.width;
  if (bad) held = 0;
  for (int32_t j = from; j < held; j += step) {
    int32_t id = a.table[int64_t(r) * a.stride + j];
    if (uint32_t(id) >= uint32_t(a.n_pages)) {
      bad = true;
    } else {
      const int32_t m = a.list[id];
      if (m < 0)
        bad = true;  // a held page that is free: its id may be another's now
      else if (id >= L)
        id = a.dst[m];
    }
    a.table_out[int64_t(r) * a.out_stride + j] = id;
  }
  if (bad) raise_err(a.err, FS_E_RANGE);
}

// Pools of few pages.  WHOLE: the counts and few rows of the table too, two for each wave.
template <bool WHOLE>
__global__ void __launch_bounds__(kBlock) k_pages_moves_few(PoolArgs a) {
  __shared__ int32_t lds[kBlock / 64];
  int32_t mine = 0, L, below = 0;
  my_pages(a, [&](int32_t, int32_t refs) { mine += __popcll(__ballot(refs > 0)); });
  int32_t rank = waves_before(mine, lds, L);
  my_pages(a, [&](int32_t p, int32_t refs) { below += __popcll(__ballot(p < L && refs > 0)); });
  int32_t all_below;
  waves_before(below, lds, all_below);
  if (threadIdx.x == 0) put_moves(a, L, all_below);
  my_pages(a, [&](int32_t p, int32_t refs) {
    const uint64_t live = __ballot(refs > 0);
    if (p < a.n_pages) place_page(a, p, refs, rank + lanes_before(live), L, all_below);
    rank += __popcll(live);
  });
  if constexpr (WHOLE) {
    __syncthreads();
    move_counts(a, L - all_below, threadIdx.x, kBlock);
    for (int32_t r = threadIdx.x >> 6; r < a.n_rows; r += kBlock / 64)
      remap_row(a, L, r, threadIdx.x & 63, 64);
  }
}

// The same for pools of many pages.
__global__ void __launch_bounds__(kBlock) k_pages_moves(PoolArgs a) {
  __shared__ int32_t lds[kBlock / 64];
  const int tid = threadIdx.x;
  int32_t before = 0, L = 0;
  for (int32_t b = tid; b < a.blocks; b += kBlock) {
    const int32_t x = a.block_sum[b];
    L += x;
    if (b < int32_t(blockIdx.x)) before += x;
  }
  before = block_total(before, lds);
  L = block_total(L, lds);
  // of the pages in use, those below L
  const int32_t lb = L / kPer;
  int32_t below = 0;
  for (int32_t b = tid; b < lb; b += kBlock) below += a.block_sum[b];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int32_t p = lb * kPer + i * kBlock + tid;
    if (p < L) below += a.refs[p] > 0;
  }
  below = block_total(below, lds);
  if (blockIdx.x == 0 && tid == 0) put_moves(a, L, below);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int32_t p = blockIdx.x * kPer + i * kBlock + tid;
    const int32_t refs = p < a.n_pages ? a.refs[p] : 0;
    const int32_t live = refs > 0;
    const int32_t rank = before + block_before(live, lds);
    before += block_total(live, lds);
    if (p < a.n_pages) place_page(a, p, refs, rank, L, below);
  }
}

// The first table_blocks work-groups, `per_row` a row, take the table, the others the counts.
__global__ void __launch_bounds__(256) k_pages_remap(PoolArgs a, int32_t table_blocks,
                                                     int32_t per_row) {
  const int32_t L = a.word[0], moves = a.word[1], b = blockIdx.x;
  const int tid = threadIdx.x;
  if (b >= table_blocks) {
    move_counts(a, moves, (b - table_blocks) * 256 + tid, (gridDim.x - table_blocks) * 256);
  } else {
    const int32_t r = b / per_row;
    remap_row(a, L, r, (b - r * per_row) * 256 + tid, per_row * 256);
  }
}

// ---- copies
struct CopyArgs {
  PageArrays arrays;
  PageShape codes, scales;
  int32_t n_layers, n_kinds, n_pages, n;
  int32_t code_parts, scale_parts;  // work-groups' shares of a page
  const int32_t *src, *dst, *count;
  int32_t *err;
};

constexpr int kUnroll = 4;  // loads of a thread under way

// Bytes by T from the pieces of one page to another's: its `part`-th 256 * kUnroll values of T.
template <class T>
__device__ inline void copy_page(char *base, const PageShape &s, int64_t from, int64_t to,
                                 int32_t part) {
  const uint32_t per = s.bytes / sizeof(T), total = s.heads * s.tokens * per;
  const uint32_t begin = uint32_t(part) * (256 * kUnroll);
  T x[kUnroll];
  int64_t at[kUnroll];
#pragma unroll
  for (int i = 0; i < kUnroll; ++i) {
    const uint32_t e = begin + i * 256 + threadIdx.x;
    at[i] = -1;
    if (e >= total) continue;
    if (per == total) {  // the page is one piece
      at[i] = int64_t(e) * sizeof(T);
    } else {
      const uint32_t piece = e / per, h = piece / s.tokens;
      at[i] = int64_t(h) * s.head_stride + int64_t(piece - h * s.tokens) * s.token_stride +
              int64_t(e - piece * per) * sizeof(T);
    }
    x[i] = *reinterpret_cast<const T *>(base + from + at[i]);
  }
#pragma unroll
  for (int i = 0; i < kUnroll; ++i)
    if (at[i] >= 0) *reinterpret_cast<T *>(base + to + at[i]) = x[i];
}

template <bool VEC_SCALES>
__global__ void __launch_bounds__(256) k_pages_copy(CopyArgs a) {
  typedef uint32_t __attribute__((ext_vector_type(4))) V;
  const int32_t n = a.count ? min(max(*a.count, 0), a.n) : a.n;
  const int32_t each = 2 * a.code_parts + (a.n_kinds > 2 ? 2 * a.scale_parts : 0);
  const int32_t per = each * a.n_layers;
  for (int64_t u = blockIdx.x; u < int64_t(n) * per; u += gridDim.x) {
    const int32_t i = int32_t(u / per), r = int32_t(u - int64_t(i) * per);
    const int32_t src = a.src[i], dst = a.dst[i];
    if (src == -1 && dst == -1) continue;
    if (uint32_t(src) >= uint32_t(a.n_pages) || uint32_t(dst) >= uint32_t(a.n_pages)) {
      if (r == 0 && threadIdx.x == 0) raise_err(a.err, FS_E_RANGE);
      continue;
    }
    const int32_t layer = r / each, w = r - layer * each;
    if (w < 2 * a.code_parts) {
      const int32_t kind = w >= a.code_parts;
      copy_page<V>(a.arrays.at[layer][kind], a.codes, src * a.codes.page_stride,
                   dst * a.codes.page_stride, w - kind * a.code_parts);
    } else {
      const int32_t ws = w - 2 * a.code_parts, kind = ws >= a.scale_parts;
      char *base = a.arrays.at[layer][2 + kind];
      const int64_t from = src * a.scales.page_stride, to = dst * a.scales.page_stride;
      if constexpr (VEC_SCALES)
        copy_page<V>(base, a.scales, from, to, ws - kind * a.scale_parts);
      else
        copy_page<uint8_t>(base, a.scales, from, to, ws - kind * a.scale_parts);
    }
  }
}

size_t round256(size_t x) { return (x + 255) / 256 * 256; }
int32_t page_blocks(const fs_pages *p) { return (p->n_pages + kPer - 1) / kPer; }

PoolArgs pool_args(const fs_pages *p, int32_t n, void *ws, int32_t *err) {
  PoolArgs a = {};
  a.n_pages = p->n_pages;
  a.page_shift = __builtin_ctz(unsigned(p->page_size));
  a.n_rows = p->n_rows;
  a.width = p->width;
  a.refs = p->refs;
  a.table = p->table;
  a.held = p->held;
  a.stride = p->table_stride;
  a.n = n;
  a.blocks = page_blocks(p);
  a.err = err;
  char *at = static_cast<char *>(ws);
  auto take = [&](size_t values) {
    int32_t *x = reinterpret_cast<int32_t *>(at);
    at += round256(values * 4);
    return x;
  };
  a.word = take(2);
  a.block_sum = take(a.blocks);
  a.list = take(p->n_pages);
  a.claim = take(p->n_rows);
  a.first = take(n);
  return a;
}

}  // namespace

size_t pages_workspace_bytes(const fs_pages *p, int32_t n) {
  return 256 + round256(size_t(page_blocks(p)) * 4) + round256(size_t(p->n_pages) * 4) +
         round256(size_t(p->n_rows) * 4) + round256(size_t(n) * 4);
}

hipError_t launch_pages_free(const fs_pages *p, int32_t n, const int32_t *rows, int32_t *err,
                             hipStream_t stream) {
  PoolArgs a = pool_args(p, 0, nullptr, err);
  a.n = n;
  a.rows = rows;
  hipLaunchKernelGGL(k_pages_free, dim3(n < kFreeBlocks ? n : kFreeBlocks), dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_pages_fork(const fs_pages *p, int32_t n, const int32_t *parent,
                             const int32_t *child, const int32_t *shared, const int32_t *room,
                             int32_t *src, int32_t *dst, void *ws, int32_t *err,
                             hipStream_t stream) {
  PoolArgs a = pool_args(p, n, ws, err);
  a.parent = parent;
  a.child = child;
  a.shared = shared;
  a.room = room;
  a.src = src;
  a.dst = dst;
  const int64_t most = int64_t(n) * p->width;
  a.most = int32_t(most < p->n_pages ? most : p->n_pages);
  if (p->n_pages <= kFewPages && n <= kSomeForks) {
    if (n <= kFewForks) {
      hipLaunchKernelGGL((k_pages_plan<true>), dim3(1), dim3(kBlock), 0, stream, a);
      return hipGetLastError();
    }
    hipLaunchKernelGGL((k_pages_plan<false>), dim3(1), dim3(kBlock), 0, stream, a);
  } else {
    const int32_t checks = (n + kBlock / 64 - 1) / (kBlock / 64);
    hipLaunchKernelGGL((k_pages_count<false>), dim3(a.blocks + checks), dim3(kBlock), 0, stream, a);
    hipLaunchKernelGGL(k_pages_list, dim3(a.blocks + 1), dim3(kBlock), 0, stream, a);
  }
  hipLaunchKernelGGL(k_pages_fork, dim3(n), dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const fs_pages *p, int32_t *refs_out, int32_t *table_out,
                                int64_t table_out_stride, int32_t *src, int32_t *dst,
                                int32_t *count, void *ws, int32_t *err, hipStream_t stream) {
  PoolArgs a = pool_args(p, 0, ws, err);
  a.refs_out = refs_out;
  a.table_out = table_out;
  a.out_stride = table_out_stride;
  a.src = src;
  a.dst = dst;
  a.count = count;
  if (p->n_pages <= kFewPages) {
    if (p->n_rows <= kFewForks && p->width <= 1024) {
      hipLaunchKernelGGL((k_pages_moves_few<true>), dim3(1), dim3(kBlock), 0, stream, a);
      return hipGetLastError();
    }
    hipLaunchKernelGGL((k_pages_moves_few<false>), dim3(1), dim3(kBlock), 0, stream, a);
  } else {
    hipLaunchKernelGGL((k_pages_count<true>), dim3(a.blocks), dim3(kBlock), 0, stream, a);
    hipLaunchKernelGGL(k_pages_moves, dim3(a.blocks), dim3(kBlock), 0, stream, a);
  }
  const int32_t per_row = p->width <= 1024 ? 1 : p->width <= 65536 ? (p->width + 1023) / 1024 : 64;
  const int32_t table_blocks = p->n_rows * per_row;
  const int32_t moves = p->n_pages / 2 / 256 + 1;
  hipLaunchKernelGGL(k_pages_remap, dim3(table_blocks + (moves < 256 ? moves : 256)), dim3(256), 0,
                     stream, a, table_blocks, per_row);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const PageArrays &arrays, int32_t n_layers, int32_t n_kinds,
                             const PageShape &codes, const PageShape &scales, int32_t n_pages,
                             int32_t n, const int32_t *src, const int32_t *dst,
                             const int32_t *count, int32_t *err, hipStream_t stream) {
  CopyArgs a = {arrays, codes, scales, n_layers, n_kinds, n_pages, n, 0, 0, src, dst, count, err};
  bool vec = true;
  auto parts = [](const PageShape &s, uint32_t unit) {
    const int64_t units = int64_t(s.heads) * s.tokens * (s.bytes / unit);
    return int32_t((units + 256 * kUnroll - 1) / (256 * kUnroll));
  };
  a.code_parts = parts(codes, 16);
  if (n_kinds > 2) {
    int64_t all = scales.page_stride | scales.bytes | scales.head_stride | scales.token_stride;
    for (int32_t i = 0; i < n_layers; ++i)
      all |= int64_t(reinterpret_cast<uintptr_t>(arrays.at[i][2])) |
             int64_t(reinterpret_cast<uintptr_t>(arrays.at[i][3]));
    vec = all % 16 == 0;
    a.scale_parts = parts(scales, vec ? 16 : 1);
  }
  const int64_t units =
      int64_t(n) * n_layers * (2 * a.code_parts + (n_kinds > 2 ? 2 * a.scale_parts : 0));
  const dim3 grid(uint32_t(units < 4096 ? units : 4096)), block(256);
  if (vec)
    hipLaunchKernelGGL((k_pages_copy<true>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((k_pages_copy<false>), grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace fs
