// A linear layer for few rows (gfx950): what a token, or a serving step's tokens,
// cost is reading W once, so W is read as FP32 and split in registers, and nothing
// but the result is written.  Few columns are the same with the sides exchanged,
// Y^T = W^T X^T: "X" is then W^T, whose rows may lie along k or (kAcross) across it,
// and "W" is X.
//
// Both kernels multiply 16-row blocks of X with 16 columns of W a wave, a 32-wide
// step of k at a time: three v_mfma_f32_16x16x32_f16 per block, A_hi B_hi into one
// accumulator and A_lo B_hi + A_hi B_lo into another (the termwise order with both
// cross terms in one sum).  Where one pass over k on few columns would leave
// compute units idle, S workgroups share the k of a group of columns and write
// partial sums that a second kernel joins, always in the same order.
//
// The k that a lane's eight values of a fragment stand for only has to be the same
// for X and W.  Rows of W along k ("nk"): quads 4 g .. and 16 + 4 g .. of the step
// for lane group g, so that one 16-byte load of a wave covers 64 adjacent bytes of
// 16 rows.  Rows along n ("kn"): k = 8 g + e, one load per k.
#include <algorithm>

#include "activation.h"
#include "gemm_common.h"
#include "layers.h"

namespace sgc {
namespace {

constexpr int kStep = 32;  // k per MFMA
constexpr int kBlockRows = 16;

typedef float floatx4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef _Float16 half2 __attribute__((ext_vector_type(2)));

// Eight values and their split (Sec. 3.3): hi = fl16(v), lo = fl16((v - hi) s).
struct Values {
  float v[8];
  // Times 2^shift, for a gradient.
  template <bool kGrad>
  __device__ __forceinline__ Values shifted(int shift) const {
    Values x = *this;
    if constexpr (kGrad) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x.v[e] = __builtin_ldexpf(x.v[e], shift);
    }
    return x;
  }
  __device__ __forceinline__ void split(float s, half8& hi, half8& lo) const {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const floatx2 x = {v[e], v[e + 1]};
      const half2 h = __builtin_convertvector(x, half2);
      const floatx2 r = {x[0] - static_cast<float>(h[0]), x[1] - static_cast<float>(h[1])};
      const floatx2 rs = {r[0] * s, r[1] * s};
      const half2 l = __builtin_convertvector(rs, half2);
      hi[e] = h[0], hi[e + 1] = h[1];
      lo[e] = l[0], lo[e + 1] = l[1];
    }
  }
};

// First k of quad q (0, 1) of lane group g, within a step.
template <bool kNk>
__device__ __forceinline__ int quad_k(int g, int q) {
  return kNk ? 16 * q + 4 * g : 8 * g + 4 * q;
}

// A row's eight values of step k0; past `k_end` zeros (only where kTail).
template <bool kNk, bool kTail>
__device__ __forceinline__ void load_along(const float* row, int64_t k0, int64_t k_end, int g,
                                           Values& out) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int64_t k = k0 + quad_k<kNk>(g, q);
    if constexpr (kTail) {
#pragma unroll
      for (int e = 0; e < 4; ++e) out.v[4 * q + e] = k + e < k_end ? row[k + e] : 0.0f;
    } else {
      const floatx4_any x = *reinterpret_cast<const floatx4_any*>(row + k);
#pragma unroll
      for (int e = 0; e < 4; ++e) out.v[4 * q + e] = x[e];
    }
  }
}

// kn: a column's eight values of step k0.
template <bool kTail>
__device__ __forceinline__ void load_across(const float* col, int64_t ldw, int64_t k0,
                                            int64_t k_end, int g, Values& out) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int64_t k = k0 + 8 * g + e;
    out.v[e] = !kTail || k < k_end ? col[k * ldw] : 0.0f;
  }
}

// Rows along n: eight values of step k0 of one column, each `ld` apart, at the k
// that kNk gives them.
template <bool kNk, bool kTail>
__device__ __forceinline__ void load_strided(const float* col, int64_t ld, int64_t k0,
                                             int64_t k_end, int g, Values& out) {
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t k = k0 + quad_k<kNk>(g, q) + e;
      out.v[4 * q + e] = !kTail || k < k_end ? col[k * ld] : 0.0f;
    }
}

struct RowsArgs {
  LinearArgs a;
  const int* row_shift;  // of a gradient's rows, or null
  bool swapped;  // Y^T = W^T X^T: entry (i, j) is row j, column i of Y
  float inv_s;
  int groups;      // of columns
  int splits;      // workgroups that share a group's k
  float* partial;  // splits x M x N, where splits > 1
};

// Stores the result of row i, column j of Y.
__device__ __forceinline__ void finish(const RowsArgs& g, int64_t i, int64_t j, float z) {
  float* const y = g.a.y + i * g.a.ldy + j;
  const Epilogue& e = g.a.e;
  if (g.row_shift) {
    *y = __builtin_ldexpf(z, -g.row_shift[i]);
    return;
  }
  if (e.bias) z += e.bias[j];
  if (e.z) e.z[i * e.ldz + j] = z;
  const float v = activate(e.activation, z);
  *y = e.r ? v + e.r[i * e.ldr + j] : v;
}

// Sum v of this split for entry (i, j): the result, or a partial sum.
__device__ __forceinline__ void store(const RowsArgs& g, int split, int64_t i, int64_t j, float v) {
  if (g.splits == 1)
    finish(g, g.swapped ? j : i, g.swapped ? i : j, v);
  else
    g.partial[(split * g.a.M + i) * g.a.N + j] = v;
}

// Up to 16 rows (plan_rows): the waves of a workgroup share 16 C columns and take the
// steps of k in turn, and add their sums in LDS.  Where W's rows are along k they
// read 2 KiB of each of those rows in line together.  1 x 8192 x 4096: 25.7 us, 5.2
// TB/s (64 columns a workgroup as below 30; 8 waves 28.6; one column block 30).
constexpr int kLineWaves = 16;

template <bool kNk, int kC, bool kGrad, bool kAcross>
__global__ __launch_bounds__(64 * kLineWaves) void linear_line_kernel(RowsArgs g) {
  const LinearArgs& a = g.a;
  __shared__ float tile[kLineWaves][256 * kC];
  const int lane = threadIdx.x & 63, group = lane >> 4, l16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int index = xcd_order(blockIdx.x, gridDim.x);
  const int col_group = index / g.splits, split = index - col_group * g.splits;
  const int64_t col0 = static_cast<int64_t>(col_group) * (16 * kC);
  // Rows and columns past the end repeat the last; they are not stored.
  const int64_t row = min<int64_t>(l16, a.M - 1);
  const float* const xrow = a.x + row * (kAcross ? 1 : a.ldx);
  const int shift = kGrad ? g.row_shift[row] : 0;
  const float* wcol[kC];
#pragma unroll
  for (int c = 0; c < kC; ++c)
    wcol[c] = a.w + min<int64_t>(col0 + 16 * c + l16, a.N - 1) * (kNk ? a.ldw : 1);

  struct Step {
    Values x, w[kC];
  };
  auto load = [&](int64_t step, Step& s, auto tail) {
#pragma unroll
    for (int c = 0; c < kC; ++c)
      if constexpr (kNk)
        load_along<true, tail.value>(wcol[c], step * kStep, a.K, group, s.w[c]);
      else
        load_across<tail.value>(wcol[c], a.ldw, step * kStep, a.K, group, s.w[c]);
    if constexpr (kAcross)
      load_strided<kNk, tail.value>(xrow, a.ldx, step * kStep, a.K, group, s.x);
    else
      load_along<kNk, tail.value>(xrow, step * kStep, a.K, group, s.x);
  };
  floatx4 hh[kC], cross[kC];
#pragma unroll
  for (int c = 0; c < kC; ++c) hh[c] = cross[c] = floatx4{};
  auto multiply = [&](const Step& s) {
    half8 xh, xl;
    s.x.template shifted<kGrad>(shift).split(a.scale, xh, xl);
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      half8 wh, wl;
      s.w[c].split(a.scale, wh, wl);
      hh[c] = mfma16(xh, wh, hh[c]);
      cross[c] = mfma16(xl, wh, cross[c]);
      cross[c] = mfma16(xh, wl, cross[c]);
    }
  };

  // Whole steps t, t + stride, ... and, last, the one that K ends in.  The next
  // step's loads are issued before this one is multiplied.
  const int64_t whole = a.K / kStep, stride = static_cast<int64_t>(g.splits) * kLineWaves;
  int64_t t = static_cast<int64_t>(split) * kLineWaves + wave;
  const std::false_type no;
  const std::true_type yes;
  if (t < whole) {
    Step s0, s1;
    load(t, s0, no);
    while (true) {
      if (t + stride < whole) load(t + stride, s1, no);
      multiply(s0);
      t += stride;
      if (t >= whole) break;
      if (t + stride < whole) load(t + stride, s0, no);
      multiply(s1);
      t += stride;
      if (t >= whole) break;
    }
  }
  if (t == whole && whole * kStep < a.K) {
    Step s;
    load(t, s, yes);
    multiply(s);
  }

  constexpr int kWidth = 16 * kC;
#pragma unroll
  for (int c = 0; c < kC; ++c)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      tile[wave][(4 * group + r) * kWidth + 16 * c + l16] =
          __builtin_fmaf(cross[c][r], g.inv_s, hh[c][r]);
  __syncthreads();
  for (int q = threadIdx.x; q < 16 * kWidth; q += 64 * kLineWaves) {
    const int64_t i = q / kWidth, j = col0 + q % kWidth;
    if (i >= a.M || j >= a.N) continue;
    float v = tile[0][q];
#pragma unroll
    for (int w = 1; w < kLineWaves; ++w) v += tile[w][q];
    store(g, split, i, j, v);
  }
}

// Other layouts and more rows: 64 columns a workgroup, 16 a wave, up to 96 rows, a
// stretch of k per workgroup.  X is split once per workgroup, 64 k at a time, into
// LDS in the order of the fragments (a wave reads 1 KiB in line), W in the
// registers of the wave that multiplies it; the next two stretches of W and the
// next of X are on their way meanwhile.  Without the sharing, X's loads and its
// split in every wave outweighed W's: 64 x 8192 x 8192 146 us, so 76 (3.5 TB/s); 48
// x 4096 x 4096 33 and 26, of which the join is 4.  Half of a wave's time is still
// waiting for W: 128 k at a time and two workgroups per compute unit instead of
// three: 80-85 us; 32 k and four: 70-79.
constexpr int kTileWaves = 4, kTileCols = 16 * kTileWaves;
constexpr int kChunkSteps = 2, kChunkK = kChunkSteps * kStep;

template <bool kNk, int kR, bool kGrad, bool kAcross>
__global__ __launch_bounds__(64 * kTileWaves, kR > (kAcross ? 4 : 5) ? 2 : 3)
void linear_rows_tile_kernel(RowsArgs g) {
  const LinearArgs& a = g.a;
  constexpr int kUnits = kChunkSteps * kR;  // fragments of a chunk of X, of each plane
  extern __shared__ __align__(16) half8 frags[];  // 2 x kUnits x 2 x 64
  const int lane = threadIdx.x & 63, group = lane >> 4, l16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int index = xcd_order(blockIdx.x, gridDim.x);
  const int col_group = index / g.splits, split = index - col_group * g.splits;
  const int64_t row0 = static_cast<int64_t>(blockIdx.y) * (kBlockRows * kR);
  const int64_t col = static_cast<int64_t>(col_group) * kTileCols + 16 * wave + l16;
  // Whole chunks c0 .. c1 - 1, and for the last split the one that K ends in.
  const int64_t chunks = a.K / kChunkK;
  const int64_t c0 = chunks * split / g.splits, c1 = chunks * (split + 1) / g.splits;

  const float* const wcol = a.w + min<int64_t>(col, a.N - 1) * (kNk ? a.ldw : 1);
  // Units of X's chunk: step u / kR, row block u % kR.  The waves take them in turn,
  // the last one again where there are fewer.
  constexpr int kPer = (kUnits + kTileWaves - 1) / kTileWaves;
  int unit[kPer], shift[kPer];
  const float* xrow[kPer];
#pragma unroll
  for (int n = 0; n < kPer; ++n) {
    unit[n] = min(wave + kTileWaves * n, kUnits - 1);
    const int64_t row = min<int64_t>(row0 + 16 * (unit[n] % kR) + l16, a.M - 1);
    xrow[n] = a.x + row * (kAcross ? 1 : a.ldx);
    shift[n] = kGrad ? g.row_shift[row] : 0;
  }

  Values w[2][kChunkSteps], x[kPer];
  auto load_w = [&](int64_t c, int st, Values& to, auto tail) {
    const int64_t k0 = c * kChunkK + st * kStep;
    if constexpr (kNk)
      load_along<true, tail.value>(wcol, k0, a.K, group, to);
    else
      load_across<tail.value>(wcol, a.ldw, k0, a.K, group, to);
  };
  auto load_x = [&](int64_t c, auto tail) {
#pragma unroll
    for (int n = 0; n < kPer; ++n) {
      const int64_t k0 = c * kChunkK + unit[n] / kR * kStep;
      if constexpr (kAcross)
        load_strided<kNk, tail.value>(xrow[n], a.ldx, k0, a.K, group, x[n]);
      else
        load_along<kNk, tail.value>(xrow[n], k0, a.K, group, x[n]);
    }
  };
  auto store_x = [&](int slot) {
#pragma unroll
    for (int n = 0; n < kPer; ++n) {
      half8 hi, lo;
      x[n].template shifted<kGrad>(shift[n]).split(a.scale, hi, lo);
      half8* const at = frags + ((slot * kUnits + unit[n]) * 2) * 64 + lane;
      at[0] = hi;
      at[64] = lo;
    }
  };
  floatx4 hh[kR], cross[kR];
#pragma unroll
  for (int i = 0; i < kR; ++i) hh[i] = cross[i] = floatx4{};
  const std::false_type no;
  const std::true_type yes;
  // The products of a chunk; each step's registers take the loads of chunk `ahead`
  // as soon as they are split (kAhead).
  auto multiply = [&](Values (&v)[kChunkSteps], int slot, int64_t ahead, auto more) {
#pragma unroll
    for (int st = 0; st < kChunkSteps; ++st) {
      half8 wh, wl;
      v[st].split(a.scale, wh, wl);
      if constexpr (more.value) load_w(ahead, st, v[st], no);
#pragma unroll
      for (int i = 0; i < kR; ++i) {
        const half8* const at = frags + ((slot * kUnits + st * kR + i) * 2) * 64 + lane;
        const half8 xh = at[0], xl = at[64];
        hh[i] = mfma16(xh, wh, hh[i]);
        cross[i] = mfma16(xl, wh, cross[i]);
        cross[i] = mfma16(xh, wl, cross[i]);
      }
    }
  };
  // Chunk c, whose W is in w[slot] and whose X in LDS slot `slot`.  The other slot
  // is written after every wave has read chunk c - 1 there, and read after the
  // barrier.
  auto turn = [&](int64_t c, int slot, Values (&now)[kChunkSteps], auto more_x, auto more_w) {
    if constexpr (more_x.value) load_x(c + 1, no);
    multiply(now, slot, c + 2, more_w);
    if constexpr (more_x.value) store_x(slot ^ 1);
    __syncthreads();
  };
  if (c0 < c1) {
    load_x(c0, no);
#pragma unroll
    for (int st = 0; st < kChunkSteps; ++st) load_w(c0, st, w[0][st], no);
    if (c0 + 1 < c1) {
#pragma unroll
      for (int st = 0; st < kChunkSteps; ++st) load_w(c0 + 1, st, w[1][st], no);
    }
    store_x(0);
    __syncthreads();
    int64_t c = c0;
    for (; c + 3 < c1; c += 2) {
      turn(c, 0, w[0], yes, yes);
      turn(c + 1, 1, w[1], yes, yes);
    }
    // One to three are left; w holds the first two of them.
    if (c + 3 == c1) {
      turn(c, 0, w[0], yes, yes);
      turn(c + 1, 1, w[1], yes, no);
      turn(c + 2, 0, w[0], no, no);
    } else if (c + 2 == c1) {
      turn(c, 0, w[0], yes, no);
      turn(c + 1, 1, w[1], no, no);
    } else {
      turn(c, 0, w[0], no, no);
    }
  }
  if (split == g.splits - 1 && chunks * kChunkK < a.K) {
    load_x(chunks, yes);
#pragma unroll
    for (int st = 0; st < kChunkSteps; ++st) load_w(chunks, st, w[0][st], yes);
    store_x(0);  // after the barrier of the turn before
    __syncthreads();
    multiply(w[0], 0, 0, no);
  }
  if (col >= a.N) return;
#pragma unroll
  for (int i = 0; i < kR; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t row = row0 + 16 * i + 4 * group + r;
      if (row >= a.M) continue;
      store(g, split, row, col, __builtin_fmaf(cross[i][r], g.inv_s, hh[i][r]));
    }
}

__global__ __launch_bounds__(256) void linear_join_kernel(RowsArgs g) {
  const LinearArgs& a = g.a;
  const int64_t q = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (q >= a.M * a.N) return;
  const int64_t i = q / a.N, j = q - i * a.N;
  float v = 0.0f;
#pragma unroll 4
  for (int s = 0; s < g.splits; ++s) v += g.partial[s * a.M * a.N + q];
  finish(g, g.swapped ? j : i, g.swapped ? i : j, v);
}

// out = L^T R of matrices with few rows: a weight's gradient of few rows is bound by
// writing it, so the operands stay FP32 and nothing is split.  A workgroup has 64 x 256
// entries: its columns of L and R in LDS, 16 rows and four adjacent columns a thread,
// whole rows of 1 KiB a wave's store.  8192 x 4096 of one row 22.6 us (5.9 TB/s); 8064 x
// 7334 of 17 rows 65, split and by the wide tiles' products 90; of 32 rows 93 and 90, as
// the FMAs, which do not overlap the stores, pass them.
constexpr int kOuterThreads = 256, kOuterTileRows = 64, kOuterTileCols = 256;

__global__ __launch_bounds__(kOuterThreads) void linear_outer_kernel(OuterArgs g, int64_t strips,
                                                                     int64_t tiles) {
  __shared__ __align__(16) float left[kOuterRows][kOuterTileRows];
  __shared__ __align__(16) float right[kOuterRows][kOuterTileCols];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  auto value = [&](const OuterSide& s, int64_t m, int64_t j) {
    if (j >= s.cols) return 0.0f;
    const float v = s.p[m * s.ld + j];
    return s.z ? v * activate_grad(g.activation, s.z[m * s.ldz + j]) : v;
  };
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t i0 = tile / strips * kOuterTileRows, j0 = tile % strips * kOuterTileCols;
    for (int q = t; q < g.M * kOuterTileRows; q += kOuterThreads)
      left[q / kOuterTileRows][q % kOuterTileRows] =
          value(g.left, q / kOuterTileRows, i0 + q % kOuterTileRows);
#pragma unroll 4
    for (int m = 0; m < g.M; ++m) right[m][t] = value(g.right, m, j0 + t);
    __syncthreads();
    floatx4 acc[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = floatx4{};
    for (int m = 0; m < g.M; ++m) {
      const floatx4 r = *reinterpret_cast<const floatx4*>(&right[m][4 * lane]);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const floatx4 l = *reinterpret_cast<const floatx4*>(&left[m][16 * wave + 4 * q]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            acc[4 * q + e][c] = __builtin_fmaf(l[e], r[c], acc[4 * q + e][c]);
      }
    }
    const int64_t j = j0 + 4 * lane;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int64_t row = i0 + 16 * wave + i;
      if (row >= g.left.cols) break;
      float* const at = g.out + row * g.ldo + j;
      if (j + 3 < g.right.cols) {
        *reinterpret_cast<floatx4_any*>(at) = acc[i];
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (j + c < g.right.cols) at[c] = acc[i][c];
      }
    }
    __syncthreads();  // the tile's LDS is read before the next's is written
  }
}

struct RowsPlan {
  bool line;  // linear_line_kernel
  int blocks;  // 16-row blocks (tile) or 16-column blocks (line) of a workgroup
  int groups, row_groups, splits;
};

RowsPlan plan_rows(int64_t M, int64_t N, int64_t K, bool transpose_w) {
  RowsPlan p{};
  // Rows of W along n: 16 columns are half a cache line, which costs large weights
  // more than the tiles' join (1 x 8192 x 8192 73 us, tiles 51; 16 x 4096 x 4096 22.6
  // and 20.3) and small ones less (1 x 2048 x 2048 8.9 and 11.7, 512 x 512 9.0 and
  // 11.6, 1024 x 4096 11.8 and 11.6).
  p.line = M <= kBlockRows && (transpose_w || N * K <= (int64_t{1} << 22));
  int64_t most, fill;
  if (p.line) {
    // A compute unit holds one workgroup, and a round of them takes 12 us with one
    // block of columns and 21 with two (K = 4096): 1 x 6144 25.0 and 21.3 us, 8192 29.2
    // and 25.8, 11008 37.5 and 42.4, 14336 48.4 and 44.0.
    const int64_t one = (N + 4095) / 4096, two = (N + 8191) / 8192;
    p.blocks = transpose_w && 7 * two <= 4 * one ? 2 : 1;
    p.groups = static_cast<int>((N + 16 * p.blocks - 1) / (16 * p.blocks));
    p.row_groups = 1;
    most = K / kStep / (4 * kLineWaves);  // four steps a wave at least
    fill = 256;
  } else {
    // 65 to 96 rows in one group read W once and not twice: 65 x 8192 x 8192 kn 108 us in
    // two, 83 so; 96 x 4096 x 4096 nk 39 and 32; few columns 10265 x 84 x 6848 137 and 88.
    // Small kn weights lose a little (80 x 2048 x 2048 12.6 and 13.3), 128 rows in one
    // group (registers) more.
    const bool six = M > 64 && M <= 96 && (transpose_w || N >= 4096);
    p.blocks = static_cast<int>(std::min<int64_t>((M + kBlockRows - 1) / kBlockRows, six ? 6 : 4));
    p.row_groups = static_cast<int>((M + kBlockRows * p.blocks - 1) / (kBlockRows * p.blocks));
    // The groups even.
    const int64_t even = kBlockRows * static_cast<int64_t>(p.row_groups);
    p.blocks = static_cast<int>((M + even - 1) / even);
    p.groups = static_cast<int>((N + kTileCols - 1) / kTileCols);
    // The join costs 4 us, as much as four chunks of a lone workgroup.
    most = K / kChunkK > 5 ? K / kChunkK / 2 : 1;
    fill = p.blocks > 5 ? 512 : 768;  // what the registers of a compute unit hold
  }
  const int64_t want = fill / (static_cast<int64_t>(p.groups) * p.row_groups);
  p.splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({want, most, 16})));
  return p;
}

template <bool kNk, int kC, bool kGrad, bool kAcross = false>
hipError_t launch_line(const RowsArgs& g, const RowsPlan& p, hipStream_t stream) {
  hipLaunchKernelGGL((linear_line_kernel<kNk, kC, kGrad, kAcross>), dim3(p.groups * p.splits),
                     dim3(64 * kLineWaves), 0, stream, g);
  return hipGetLastError();
}

template <bool kNk, int kR, bool kGrad, bool kAcross>
hipError_t launch_tile(const RowsArgs& g, const RowsPlan& p, hipStream_t stream) {
  constexpr size_t kLds = static_cast<size_t>(2) * kChunkSteps * kR * 2 * 1024;
  static_assert(kLds <= 64 * 1024, "both chunks fit LDS without asking for more");
  hipLaunchKernelGGL((linear_rows_tile_kernel<kNk, kR, kGrad, kAcross>),
                     dim3(p.groups * p.splits, p.row_groups), dim3(64 * kTileWaves), kLds, stream,
                     g);
  return hipGetLastError();
}

template <bool kNk, bool kGrad, bool kAcross = false>
hipError_t launch_tiles(const RowsArgs& g, const RowsPlan& p, hipStream_t stream) {
  switch (p.blocks) {
    case 1: return launch_tile<kNk, 1, kGrad, kAcross>(g, p, stream);
    case 2: return launch_tile<kNk, 2, kGrad, kAcross>(g, p, stream);
    case 3: return launch_tile<kNk, 3, kGrad, kAcross>(g, p, stream);
    case 4: return launch_tile<kNk, 4, kGrad, kAcross>(g, p, stream);
    case 5: return launch_tile<kNk, 5, kGrad, kAcross>(g, p, stream);
    default: return launch_tile<kNk, 6, kGrad, kAcross>(g, p, stream);
  }
}

template <bool kGrad>
hipError_t launch_plan(const RowsArgs& g, const RowsPlan& p, hipStream_t stream) {
  if (p.line)
    return !g.a.transpose_w ? launch_line<false, 1, kGrad>(g, p, stream)
           : p.blocks == 1  ? launch_line<true, 1, kGrad>(g, p, stream)
                            : launch_line<true, 2, kGrad>(g, p, stream);
  return g.a.transpose_w ? launch_tiles<true, kGrad>(g, p, stream)
                         : launch_tiles<false, kGrad>(g, p, stream);
}

// The join, where sums were left for one.
hipError_t launch_join(const RowsArgs& g, hipStream_t stream) {
  if (g.splits == 1) return hipSuccess;
  hipLaunchKernelGGL(linear_join_kernel,
                     dim3(static_cast<unsigned>((g.a.M * g.a.N + 255) / 256)), dim3(256), 0,
                     stream, g);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_outer(const OuterArgs& g, hipStream_t stream) {
  const int64_t strips = (g.right.cols + kOuterTileCols - 1) / kOuterTileCols;
  const int64_t tiles = (g.left.cols + kOuterTileRows - 1) / kOuterTileRows * strips;
  hipLaunchKernelGGL(linear_outer_kernel,
                     dim3(static_cast<unsigned>(std::min<int64_t>(tiles, int64_t{1} << 22))),
                     dim3(kOuterThreads), 0, stream, g, strips, tiles);
  return hipGetLastError();
}

size_t linear_rows_ws(int64_t M, int64_t N, int64_t K) {
  const int splits = std::max(plan_rows(M, N, K, false).splits, plan_rows(M, N, K, true).splits);
  // One block at least, so that every product needs a workspace.
  return static_cast<size_t>(round_up(splits > 1 ? splits * M * N * 4 : 1, 256));
}

hipError_t launch_linear_rows(const LinearArgs& a, const int* row_shift, void* ws,
                              hipStream_t stream) {
  const RowsPlan p = plan_rows(a.M, a.N, a.K, a.transpose_w);
  const RowsArgs g{a, row_shift, false, 1.0f / a.scale, p.groups, p.splits,
                   static_cast<float*>(ws)};
  const hipError_t e =
      row_shift ? launch_plan<true>(g, p, stream) : launch_plan<false>(g, p, stream);
  return e == hipSuccess ? launch_join(g, stream) : e;
}

hipError_t launch_linear_columns(const LinearArgs& a, void* ws, hipStream_t stream) {
  LinearArgs t = a;
  t.M = a.N, t.N = a.M;
  t.x = a.w, t.ldx = a.ldw;
  t.w = a.x, t.ldw = a.ldx, t.transpose_w = true;
  const RowsPlan p = plan_rows(t.M, t.N, t.K, true);
  const RowsArgs g{t, nullptr, true, 1.0f / a.scale, p.groups, p.splits,
                   static_cast<float*>(ws)};
  const hipError_t e =
      a.transpose_w ? launch_plan<false>(g, p, stream)
      : !p.line     ? launch_tiles<true, false, true>(g, p, stream)
      : p.blocks == 1 ? launch_line<true, 1, false, true>(g, p, stream)
                      : launch_line<true, 2, false, true>(g, p, stream);
  return e == hipSuccess ? launch_join(g, stream) : e;
}

}  // namespace sgc
