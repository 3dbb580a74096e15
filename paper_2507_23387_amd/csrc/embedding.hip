// Embedding lookup and its gradient (gfx950).
//
// Forward: y_i = scale W[id_i], one rounding from 32 bits to the table's type.
// Backward: dW_v = scale sum of dy_i over the i with id_i = v.  The positions are
// sorted by id first, those of one id in the order they came, and runs of equal ids
// are summed in registers, so that nothing is added by atomics: the order of every
// sum depends on the ids alone.
#include <algorithm>

#include "elem.h"
#include "layers.h"

namespace sgc {
namespace {

constexpr int kThreads = 256;

// A row's pieces by `lanes` threads (a power of two), four pieces in flight each.  HBM
// bounds it, or for few rows the two dependent loads' latency.
template <int kDtype>
__global__ __launch_bounds__(kThreads) void embedding_kernel(EmbeddingArgs a, int lanes,
                                                             int64_t groups) {
  using L = Elem<kDtype>;
  typedef typename L::T T;
  constexpr int kU = 4;
  const int sub = threadIdx.x / lanes, l = threadIdx.x % lanes, per = kThreads / lanes;
  const int cols = static_cast<int>(a.cols);
  for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
    const int64_t i = g * per + sub;
    if (i >= a.n) continue;
    const int64_t id = id_at(a.ids, i);
    T* const y = static_cast<T*>(a.y) + i * a.ldy;
    if (id < 0 || id >= a.vocab) {
      float v[L::kE];
#pragma unroll
      for (int e = 0; e < L::kE; ++e) v[e] = id < 0 ? 0.0f : __builtin_nanf("");
      for (int64_t j = l * L::kE; j < cols; j += lanes * L::kE)
        store_piece<kDtype>(y, static_cast<int>(j), cols, v);
      continue;
    }
    const T* const w = static_cast<const T*>(a.w) + id * a.ldw;
    for (int64_t j0 = l * L::kE; j0 < cols; j0 += kU * lanes * L::kE) {
      float v[kU][L::kE];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int64_t j = j0 + u * lanes * L::kE;
        if (j < cols) load_piece<kDtype>(w, static_cast<int>(j), cols, v[u]);
      }
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int64_t j = j0 + u * lanes * L::kE;
#pragma unroll
        for (int e = 0; e < L::kE; ++e) v[u][e] *= a.scale;
        if (j < cols) store_piece<kDtype>(y, static_cast<int>(j), cols, v[u]);
      }
    }
  }
}

// --- the positions in order of their ids -------------------------------------------
//
// A stable radix sort, `bits` of the key a pass.  A workgroup takes 4096 positions in
// order, a wave 256 of them, 64 at a time: lanes of equal digits find each other by
// ballots, so that a position's rank among its wave's is known without atomics.

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kSortRounds = 4, kSortItems = kSortThreads * kSortRounds;
constexpr int kDigitBits = 9, kBins = 1 << kDigitBits;

struct Sorted {
  uint32_t* keys;
  uint32_t* at;
};
struct SortPass {
  int64_t n;
  int shift, bits;
  uint32_t blocks;
  uint32_t* counts;  // kBins x blocks, bin by bin
  uint32_t* totals;  // of the bins; null: the scatter adds the counts up itself
};

// The key of position i: its id, or `vocab`, past all of them, where that is none.
__device__ __forceinline__ uint32_t key_of(const Ids& ids, int64_t vocab, int64_t i) {
  const int64_t id = id_at(ids, i);
  return static_cast<uint32_t>(id < 0 || id >= vocab ? vocab : id);
}

// Ranks of a workgroup's items by digit among those of the same wave; waves[w][d] is
// the number of wave w's items with digit d.  `live`: the item exists.
__device__ __forceinline__ void rank_items(const uint32_t (&digit)[kSortRounds],
                                           const bool (&live)[kSortRounds], int bits,
                                           uint16_t (*waves)[kBins],
                                           uint32_t (&rank)[kSortRounds]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int q = threadIdx.x; q < kSortWaves * kBins; q += kSortThreads) waves[0][q] = 0;
  __syncthreads();
  volatile uint16_t* const mine = waves[wave];
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    uint64_t peers = __ballot(live[r]);
    for (int b = 0; b < bits; ++b) {
      const bool set = digit[r] >> b & 1;
      const uint64_t with = __ballot(set);
      peers &= set ? with : ~with;
    }
    const uint64_t before = peers & ((uint64_t{1} << lane) - 1);
    const uint32_t seen = mine[digit[r]];
    rank[r] = seen + __builtin_popcountll(before);
    // A wave's LDS accesses are in order: every lane has read before one writes.
    if (live[r] && before == 0)
      mine[digit[r]] = static_cast<uint16_t>(seen + __builtin_popcountll(peers));
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
}

// waves[w][d] becomes the number of items with digit d in the waves before w, the
// result, for thread d < kBins, of all.
__device__ __forceinline__ uint32_t sum_waves(uint16_t (*waves)[kBins]) {
  uint32_t sum = 0;
  if (threadIdx.x < kBins) {
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const uint16_t c = waves[w][threadIdx.x];
      waves[w][threadIdx.x] = static_cast<uint16_t>(sum);
      sum += c;
    }
  }
  return sum;
}

// first[d], d < kBins: the sum of `count` of the threads before d.
__device__ __forceinline__ void scan_bins(uint32_t count, uint32_t* first) {
  __shared__ uint32_t wave_sums[kBins / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t sum = threadIdx.x < kBins ? count : 0;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t o = __shfl_up(sum, d);
    if (lane >= d) sum += o;
  }
  if (threadIdx.x < kBins && lane == 63) wave_sums[wave] = sum;
  __syncthreads();
  if (threadIdx.x < kBins) {
    for (int w = 0; w < wave; ++w) sum += wave_sums[w];
    first[threadIdx.x] = sum - count;
  }
  __syncthreads();
}

// A workgroup's items of one pass: from the ids (the first pass) or the pass before.
__device__ __forceinline__ void load_items(const SortPass& p, const Ids& ids, int64_t vocab,
                                           const Sorted& from, uint32_t (&key)[kSortRounds],
                                           uint32_t (&digit)[kSortRounds],
                                           bool (&live)[kSortRounds], int64_t begin) {
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const int64_t i = begin + 64 * r;
    live[r] = i < p.n;
    key[r] = !live[r] ? 0 : p.shift == 0 ? key_of(ids, vocab, i) : from.keys[i];
    digit[r] = key[r] >> p.shift & (kBins - 1);
  }
}

__device__ __forceinline__ int64_t first_item() {
  return static_cast<int64_t>(blockIdx.x) * kSortItems + (threadIdx.x >> 6) * (64 * kSortRounds) +
         (threadIdx.x & 63);
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortPass p, Ids ids,
                                                                  int64_t vocab, Sorted from) {
  __shared__ uint16_t waves[kSortWaves][kBins];
  uint32_t key[kSortRounds], digit[kSortRounds], rank[kSortRounds];
  bool live[kSortRounds];
  load_items(p, ids, vocab, from, key, digit, live, first_item());
  rank_items(digit, live, p.bits, waves, rank);
  const uint32_t sum = sum_waves(waves);
  if (threadIdx.x < kBins)
    p.counts[static_cast<int64_t>(threadIdx.x) * p.blocks + blockIdx.x] = sum;
}

// Each bin's counts become the sums of those of the blocks before; a workgroup a bin.
__global__ __launch_bounds__(kThreads) void sort_scan_kernel(SortPass p) {
  __shared__ uint32_t wave_sums[kThreads / 64];
  uint32_t* const counts = p.counts + static_cast<int64_t>(blockIdx.x) * p.blocks;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t before = 0;
  for (uint32_t b0 = 0; b0 < p.blocks; b0 += kThreads) {
    const uint32_t b = b0 + threadIdx.x, c = b < p.blocks ? counts[b] : 0;
    uint32_t sum = c;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint32_t o = __shfl_up(sum, d);
      if (lane >= d) sum += o;
    }
    if (lane == 63) wave_sums[wave] = sum;
    __syncthreads();
    uint32_t all = 0;
    for (int w = 0; w < kThreads / 64; ++w) {
      if (w == wave) sum += all;
      all += wave_sums[w];
    }
    if (b < p.blocks) counts[b] = before + sum - c;
    before += all;
    __syncthreads();  // wave_sums is read before the next turn writes it
  }
  if (threadIdx.x == 0) p.totals[blockIdx.x] = before;
}

__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(SortPass p, Ids ids,
                                                                    int64_t vocab, Sorted from,
                                                                    Sorted to) {
  __shared__ uint16_t waves[kSortWaves][kBins];
  __shared__ uint32_t first[kBins];
  uint32_t key[kSortRounds], digit[kSortRounds], rank[kSortRounds];
  bool live[kSortRounds];
  const int64_t begin = first_item();
  load_items(p, ids, vocab, from, key, digit, live, begin);
  rank_items(digit, live, p.bits, waves, rank);
  (void)sum_waves(waves);
  // This block's place in each bin: the bins before it, and the blocks before.
  uint32_t total = 0, before = 0;
  if (threadIdx.x < kBins) {
    const uint32_t* const counts = p.counts + static_cast<int64_t>(threadIdx.x) * p.blocks;
    if (p.totals) {
      total = p.totals[threadIdx.x];
      before = counts[blockIdx.x];
    } else {
      for (uint32_t b = 0; b < p.blocks; ++b) {
        const uint32_t c = counts[b];
        total += c;
        before += b < blockIdx.x ? c : 0;
      }
    }
  }
  scan_bins(total, first);
  if (threadIdx.x < kBins) first[threadIdx.x] += before;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    if (!live[r]) continue;
    const int64_t i = begin + 64 * r;
    const uint32_t d = first[digit[r]] + waves[threadIdx.x >> 6][digit[r]] + rank[r];
    to.keys[d] = key[r];
    to.at[d] = p.shift == 0 ? static_cast<uint32_t>(i) : from.at[i];
  }
}

// The median of three: k clamped to a .. b where a <= b.
__device__ __forceinline__ int clamp_of(int k, int a, int b) {
  int r;
  asm("v_med3_i32 %0, %1, %2, %3" : "=v"(r) : "v"(k), "v"(a), "v"(b));
  return r;
}

// Few positions: each one's place is the number of pairs (id, position) below its own,
// counted against all of them.  A workgroup places 64 positions, one a lane, and its
// waves share the keys, which LDS hands to all lanes at once.  Against `key`, a key k
// clamped to key - 1 .. key (before it: key .. key + 1) is one less where it counts, so
// that one instruction compares and half of one adds up; with carries there are two, and
// two waits between them.  LDS's handing out bounds it past 8192 positions: 777 4.8 us, 4096
// 8.8, 16384 24.4 (26.7 with carries; the passes above 29.4 in four launches), of which 3.5
// are the launch.
constexpr int64_t kRankItems = 16384;
constexpr int kRankChunk = 8192, kPastKeys = 0x7fffffff;
__global__ __launch_bounds__(kSortThreads) void rank_kernel(Ids ids, int64_t vocab, int n,
                                                            Sorted out) {
  __shared__ __align__(16) int keys[kRankChunk];
  __shared__ uint32_t counts[kSortWaves][64];
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i0 = blockIdx.x * 64, i = i0 + lane;
  auto key_at = [&](int j) {
    return j < n ? static_cast<int>(key_of(ids, vocab, j)) : kPastKeys;
  };
  const int key = i < n ? key_at(i) : 0;
  uint32_t below = 0;
  // Adds how many of 64 keys are below hi.
  auto count = [&](const int* group, int hi) {
    const i32x4* const at = reinterpret_cast<const i32x4*>(group);
    uint32_t sum = 0;
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      const i32x4 k = at[q];
#pragma unroll
      for (int e = 0; e < 4; e += 2)
        sum += static_cast<uint32_t>(clamp_of(k[e], hi - 1, hi)) +
               static_cast<uint32_t>(clamp_of(k[e + 1], hi - 1, hi));
    }
    below += 64 * static_cast<uint32_t>(hi) - sum;
  };
  for (int c0 = 0; c0 < n; c0 += kRankChunk) {
    const int size = min(kRankChunk, (n - c0 + 63) / 64 * 64);
    __syncthreads();  // the chunk before has been read
    for (int j = threadIdx.x; j < size; j += kSortThreads) keys[j] = key_at(c0 + j);
    __syncthreads();
    for (int g = wave * 64; g < size; g += kSortThreads) {
      if (c0 + g != i0) {
        count(keys + g, c0 + g < i0 ? key + 1 : key);
        continue;
      }
#pragma unroll 1
      for (int j = 0; j < 64; j += 4) {
        const i32x4 k = *reinterpret_cast<const i32x4*>(keys + g + j);
#pragma unroll
        for (int e = 0; e < 4; ++e) below += k[e] < key + (j + e < lane ? 1 : 0);
      }
    }
  }
  counts[wave][lane] = below;
  __syncthreads();
  if (wave != 0 || i >= n) return;
  uint32_t to = 0;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) to += counts[w][lane];
  out.keys[to] = key;
  out.at[to] = i;
}

// --- the sums -------------------------------------------------------------------------

struct SumArgs {
  EmbeddingGradArgs a;
  Sorted sorted;
  float* partial;  // chunks x 2 x cols: a chunk's first run, begun before it, and its last
  int lanes;       // threads to a chunk
  int chunk;       // positions
  int zero_rows;   // rows to a workgroup that writes zeros
  bool past;       // dW goes past the caches
  int64_t chunks;
  uint32_t sum_blocks, tiles;  // workgroups of the sums, tiles of columns
};

// The first position whose key is not below k, by a wave: 64 places at a time.
__device__ __forceinline__ int64_t wave_lower_bound(const uint32_t* keys, int64_t n, uint32_t k) {
  int64_t lo = 0, size = n;  // the answer is in lo .. lo + size
  while (size > 0) {
    const int64_t step = (size + 63) / 64, p = lo + (threadIdx.x & 63) * step;
    // The lanes' last places of their stretches: below k in a run from lane 0 on.
    const int64_t last = min(p + step, lo + size) - 1;
    const int below = __builtin_popcountll(__ballot(p < lo + size && keys[last] < k));
    const int64_t end = lo + size;
    lo = min(lo + below * step, end);
    size = min(step - 1, end - lo);
  }
  return lo;
}

// A gradient that the 256 MB last cache cannot hold goes past it, which leaves the cache
// to dy.  4096 positions of 32768 x 4096 take 126 us otherwise, with the zeros past it 112,
// with all rows 115; 16384 take 191, 186 and 156; 1048 of 112256 x 836 84, 64 and 64.  A
// smaller one stays where its reader finds it (20000 of 100000 x 512: 70, 75 past it).
// Lines that two rows share are put together in the cache (single rows of 836 values past
// it: 92).
constexpr int64_t kCacheBytes = int64_t{256} << 20;

__device__ __forceinline__ bool whole_lines(const EmbeddingGradArgs& a) {
  return (a.cols | a.lddw) % 32 == 0 && reinterpret_cast<uintptr_t>(a.dw) % 128 == 0;
}

__device__ __forceinline__ void store_grad(float* row, int j, int n, const float* v, bool past) {
  typedef Elem<kF32>::Piece Piece;
  if (past && j + 4 <= n) {
    const Piece p = {v[0], v[1], v[2], v[3]};
    __builtin_nontemporal_store(p, reinterpret_cast<Piece*>(row + j));
  } else {
    store_piece<kF32>(row, j, n, v);
  }
}

__device__ __forceinline__ void write_row(const SumArgs& g, uint32_t v, int j, int count,
                                          float* sum) {
  const EmbeddingGradArgs& a = g.a;
  float* const row = a.dw + static_cast<int64_t>(v) * a.lddw;
  const int cols = static_cast<int>(a.cols);
#pragma unroll
  for (int q = 0; q < 8; q += 4) {
    if (q >= count || j + q >= cols) break;
    if (a.accumulate) {
      float old[4];
      load_piece<kF32>(row, j + q, cols, old);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[q + e] = __builtin_fmaf(sum[q + e], a.scale, old[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[q + e] *= a.scale;
    }
    store_grad(row, j + q, cols, sum + q, g.past && whole_lines(a));
  }
}

// Rows of dW to a workgroup that looks for those without ids: 4096 values or 8 rows, and
// 4096 workgroups at most.  (8 rows of 1003 x 530 7.0 us, 32 10.8; 8 of 131072 x 64 19.4, 64
// 8.6; the call with 20000 positions of 100000 x 512 76 us in 8, 70 in 32.)
constexpr int kMostZeroRows = 64;
int zero_rows(int64_t vocab, int64_t cols) {
  int rows = 8;
  while (rows < kMostZeroRows && (2 * rows * cols <= 4096 || vocab > int64_t{4096} * rows))
    rows *= 2;
  return rows;
}

// Runs of equal ids within a chunk of sorted positions are summed by the threads that
// hold its columns, kU rows of dy in flight.  A run that goes past the chunk leaves
// its sum for the join.  The workgroups behind those of the sums write zeros to the
// rows that no position has, which a search among the keys finds.
template <int kDtype>
__global__ __launch_bounds__(kThreads) void embedding_sum_kernel(SumArgs g) {
  using L = Elem<kDtype>;
  typedef typename L::T T;
  constexpr int kE = L::kE, kU = 8;
  const EmbeddingGradArgs& a = g.a;
  const int cols = static_cast<int>(a.cols);
  if (blockIdx.x >= g.sum_blocks) {
    __shared__ bool absent[kMostZeroRows];
    __shared__ int64_t ends[2];
    const int64_t v0 = static_cast<int64_t>(blockIdx.x - g.sum_blocks) * g.zero_rows;
    const int64_t v1 = min(a.vocab, v0 + g.zero_rows);
    if (threadIdx.x < g.zero_rows) absent[threadIdx.x] = v0 + threadIdx.x < v1;
    if (threadIdx.x < 128) {
      const int wave = threadIdx.x >> 6;
      ends[wave] = wave_lower_bound(g.sorted.keys, a.n, static_cast<uint32_t>(wave ? v1 : v0));
    }
    __syncthreads();
    for (int64_t p = ends[0] + threadIdx.x; p < ends[1]; p += kThreads)
      absent[g.sorted.keys[p] - v0] = false;
    __syncthreads();
    const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const int64_t all = (v1 - v0) * a.cols;
    if (ends[0] == ends[1] && a.lddw == a.cols && all < INT32_MAX - 4) {
      // All of them, side by side.
      float* const at = a.dw + v0 * a.lddw;
      for (int64_t j = 4 * threadIdx.x; j < all; j += 4 * kThreads)
        store_grad(at, static_cast<int>(j), static_cast<int>(all), zero, g.past);
      return;
    }
    const int per = kThreads / g.lanes;
    const bool past = g.past && whole_lines(a);
    for (int r = threadIdx.x / g.lanes; r < g.zero_rows; r += per) {
      if (!absent[r]) continue;
      for (int64_t j = 4 * (threadIdx.x % g.lanes); j < cols; j += 4 * g.lanes)
        store_grad(a.dw + (v0 + r) * a.lddw, static_cast<int>(j), cols, zero, past);
    }
    return;
  }
  const int64_t group = blockIdx.x / g.tiles;
  const int tile = blockIdx.x % g.tiles;
  const int64_t c = group * (kThreads / g.lanes) + threadIdx.x / g.lanes;
  const int64_t col = (static_cast<int64_t>(tile) * g.lanes + threadIdx.x % g.lanes) * kE;
  if (c >= g.chunks || col >= cols) return;
  const int j = static_cast<int>(col);
  const uint32_t* const keys = g.sorted.keys;
  const uint32_t none = static_cast<uint32_t>(a.vocab);
  const int64_t p0 = c * g.chunk, p1 = min(a.n, p0 + g.chunk);
  // The next positions' keys and rows' numbers are asked for before this turn's rows.
  uint32_t k[kU], at[kU];
  auto ask = [&](int64_t p) {
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      k[u] = p + u < p1 ? keys[p + u] : none;
      at[u] = p + u < p1 ? g.sorted.at[p + u] : 0;
    }
  };
  ask(p0);
  const uint32_t before = p0 > 0 ? keys[p0 - 1] : none, after = p1 < a.n ? keys[p1] : none;
  uint32_t run = k[0];
  if (run == none) return;
  bool begun = before == run;  // before the chunk
  float sum[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  auto leave = [&](int which) {
    float* const to = g.partial + (2 * c + which) * a.cols;
#pragma unroll
    for (int q = 0; q < kE; q += 4)
      if (j + q < cols) store_piece<kF32>(to, j + q, cols, sum + q);
  };
  for (int64_t p = p0; p < p1; p += kU) {
    uint32_t now[kU];
    typename L::Piece v[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      now[u] = k[u];
      if (now[u] != none)
        v[u] = raw_piece<kDtype>(
            static_cast<const T*>(a.dy) + static_cast<int64_t>(at[u]) * a.lddy, j, cols);
    }
    ask(p + kU);
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      if (p + u >= p1) break;
      if (now[u] != run) {
        if (begun) leave(0);
        else write_row(g, run, j, kE, sum);
        begun = false;
        run = now[u];
        if (run == none) return;  // the last of the sorted keys
#pragma unroll
        for (int e = 0; e < kE; ++e) sum[e] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < kE; ++e) sum[e] += static_cast<float>(v[u][e]);
    }
  }
  const bool goes_on = after == run;
  if (begun) leave(0);
  else if (goes_on) leave(1);
  else write_row(g, run, j, kE, sum);
}

// Runs that begin in a chunk and go past it, a chunk a workgroup, 1024 columns: the sums
// that the chunks left, in their order.
constexpr int kJoinCols = 4 * kThreads;
__global__ __launch_bounds__(kThreads) void embedding_join_kernel(SumArgs g) {
  const EmbeddingGradArgs& a = g.a;
  const uint32_t* const keys = g.sorted.keys;
  const int cols = static_cast<int>(a.cols);
  const int64_t c = blockIdx.x, p0 = c * g.chunk, p1 = p0 + g.chunk;
  if (p1 >= a.n) return;
  const uint32_t run = keys[p1], in = keys[p1 - 1], before = p0 > 0 ? keys[p0 - 1] : ~0u;
  if (run >= a.vocab || in != run || before == run) return;
  // How many chunks begin with the run, 64 at a time.
  int64_t last = c;
  for (uint64_t more = ~uint64_t{0}; more == ~uint64_t{0};) {
    const int64_t p = (last + 1 + (threadIdx.x & 63)) * g.chunk;
    more = __ballot(p < a.n && keys[p] == run);
    last += more == ~uint64_t{0} ? 64 : __builtin_ctzll(~more);
  }
  for (int64_t j0 = static_cast<int64_t>(blockIdx.y) * kJoinCols; j0 < cols;
       j0 += static_cast<int64_t>(gridDim.y) * kJoinCols) {
    const int j = static_cast<int>(j0) + 4 * threadIdx.x;
    if (j >= cols) break;
    float sum[8] = {0.0f, 0.0f, 0.0f, 0.0f};
    load_piece<kF32>(g.partial + (2 * c + 1) * a.cols, j, cols, sum);
#pragma unroll 8
    for (int64_t d = c + 1; d <= last; ++d) {
      float v[4];
      load_piece<kF32>(g.partial + 2 * d * a.cols, j, cols, v);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += v[e];
    }
    write_row(g, run, j, 4, sum);
  }
}

// Threads to a row of `cols` values in pieces of `per`: a power of two, 16 to 256.
int row_lanes(int64_t cols, int per) {
  int lanes = 16;
  while (lanes < kThreads && static_cast<int64_t>(lanes) * per < cols) lanes *= 2;
  return lanes;
}

// Positions to a chunk: the rows of one id are added one after the other within it, and
// an id's chunks after each other, so that a long run takes as many steps of either kind
// (text's most frequent id has a tenth of all positions); but 512 workgroups, where there
// are as many chunks of 8.  Sum and join, us: 16384 x 4096 bfloat16 in chunks of 16 58 and
// 26, 32 58 and 12; 20000 x 1024 32 31 and 14, 64 41 and 7.
int chunk_length(int64_t n, int64_t cols, int per) {
  const int64_t tiles = (cols + int64_t{kThreads} * per - 1) / (int64_t{kThreads} * per);
  const int64_t groups = kThreads / row_lanes(cols, per);
  int chunk = 8;
  while (chunk < 64 && int64_t{16} * chunk * chunk < n && n * tiles / (2 * chunk * groups) >= 512)
    chunk *= 2;
  return chunk;
}

// Blocks of a pass whose counts the scatter adds up itself.
constexpr int64_t kScanBlocks = 32;

struct GradWorkspace {
  Sorted sorted[2];
  uint32_t *counts, *totals;
  float* partial;
  size_t bytes;
};

GradWorkspace carve(void* ws, int64_t n, int64_t cols) {
  char* const base = static_cast<char*>(ws);
  size_t used = 0;
  auto take = [&](int64_t bytes) {
    char* const at = base + used;
    used += static_cast<size_t>(round_up(bytes, 256));
    return at;
  };
  GradWorkspace g{};
  const int64_t blocks = (n + kSortItems - 1) / kSortItems;
  const bool passes = n > kRankItems;
  for (int s = 0; s < (passes ? 2 : 1); ++s) {
    g.sorted[s].keys = reinterpret_cast<uint32_t*>(take(4 * n));
    g.sorted[s].at = reinterpret_cast<uint32_t*>(take(4 * n));
  }
  if (passes) {
    g.counts = reinterpret_cast<uint32_t*>(take(4 * kBins * blocks));
    g.totals = reinterpret_cast<uint32_t*>(take(4 * kBins));
  }
  // The chunks of the type that has more of them.
  const int64_t chunk = std::min(chunk_length(n, cols, 4), chunk_length(n, cols, 8));
  g.partial = reinterpret_cast<float*>(take((n + chunk - 1) / chunk * 2 * cols * 4));
  g.bytes = used;
  return g;
}

hipError_t launch_sort(const EmbeddingGradArgs& a, const GradWorkspace& ws, Sorted& sorted,
                       hipStream_t stream) {
  int key_bits = 1;
  while (a.vocab >> key_bits) ++key_bits;
  sorted = ws.sorted[0];
  if (a.n <= kRankItems) {
    hipLaunchKernelGGL(rank_kernel, dim3(static_cast<unsigned>((a.n + 63) / 64)),
                       dim3(kSortThreads), 0, stream, a.ids, a.vocab, static_cast<int>(a.n),
                       sorted);
    return hipGetLastError();
  }
  const int64_t blocks = (a.n + kSortItems - 1) / kSortItems;
  SortPass p{a.n, 0, 0, static_cast<uint32_t>(blocks), ws.counts,
             blocks > kScanBlocks ? ws.totals : nullptr};
  Sorted from = ws.sorted[1];
  for (; p.shift < key_bits; p.shift += kDigitBits) {
    p.bits = std::min(kDigitBits, key_bits - p.shift);
    hipLaunchKernelGGL(sort_count_kernel, dim3(p.blocks), dim3(kSortThreads), 0, stream, p, a.ids,
                       a.vocab, from);
    if (p.totals)
      hipLaunchKernelGGL(sort_scan_kernel, dim3(kBins), dim3(kThreads), 0, stream, p);
    hipLaunchKernelGGL(sort_scatter_kernel, dim3(p.blocks), dim3(kSortThreads), 0, stream, p,
                       a.ids, a.vocab, from, sorted);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    std::swap(from, sorted);
  }
  std::swap(from, sorted);
  return hipSuccess;
}

}  // namespace

hipError_t launch_embedding(const EmbeddingArgs& a, int dtype, hipStream_t stream) {
  const int lanes = row_lanes(a.cols, dtype == kF32 ? 4 : 8);
  const int64_t per = kThreads / lanes, groups = (a.n + per - 1) / per;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(groups, int64_t{1} << 22)));
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a, lanes, groups);
    return hipGetLastError();
  };
  return dtype == kF32   ? launch(embedding_kernel<kF32>)
         : dtype == kF16 ? launch(embedding_kernel<kF16>)
                         : launch(embedding_kernel<kBF16>);
}

size_t embedding_grad_ws(int64_t n, int64_t cols) {
  return n > 0 && cols > 0 ? carve(nullptr, n, cols).bytes : 0;
}

hipError_t launch_embedding_grad(const EmbeddingGradArgs& a, int dtype, void* ws,
                                 hipStream_t stream) {
  if (a.n == 0)
    return a.accumulate ? hipSuccess : launch_zero(a.vocab, a.cols, a.dw, a.lddw, stream);
  const GradWorkspace w = carve(ws, a.n, a.cols);
  SumArgs g{};
  g.a = a;
  hipError_t err = launch_sort(a, w, g.sorted, stream);
  if (err != hipSuccess) return err;
  const int per = dtype == kF32 ? 4 : 8;
  g.partial = w.partial;
  g.lanes = row_lanes(a.cols, per);
  g.chunk = chunk_length(a.n, a.cols, per);
  g.chunks = (a.n + g.chunk - 1) / g.chunk;
  g.zero_rows = zero_rows(a.vocab, a.cols);
  g.past = a.vocab * a.cols * 4 > kCacheBytes;
  g.tiles = static_cast<uint32_t>((a.cols + int64_t{g.lanes} * per - 1) / (int64_t{g.lanes} * per));
  const int64_t groups = kThreads / g.lanes;
  const int64_t sums = (g.chunks + groups - 1) / groups * g.tiles;
  const int64_t zeros = a.accumulate ? 0 : (a.vocab + g.zero_rows - 1) / g.zero_rows;
  if ((sums + zeros) * kThreads > UINT32_MAX || g.chunks * kThreads > UINT32_MAX)
    return hipErrorInvalidValue;
  g.sum_blocks = static_cast<uint32_t>(sums);
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(sums + zeros)), dim3(kThreads), 0,
                       stream, g);
    return hipGetLastError();
  };
  err = dtype == kF32   ? launch(embedding_sum_kernel<kF32>)
        : dtype == kF16 ? launch(embedding_sum_kernel<kF16>)
                        : launch(embedding_sum_kernel<kBF16>);
  if (err != hipSuccess || g.chunks < 2) return err;
  const int64_t strips = std::min<int64_t>((a.cols + kJoinCols - 1) / kJoinCols, 65535);
  hipLaunchKernelGGL(embedding_join_kernel,
                     dim3(static_cast<unsigned>(g.chunks), static_cast<unsigned>(strips)),
                     dim3(kThreads), 0, stream, g);
  return hipGetLastError();
}

}  // namespace sgc
