// What a linear layer's products need around them (gfx950): the split of its
// operands into planes in either direction, the gradient D = dY act'(Z) with its
// column sums and its lines' largest magnitudes, and the epilogue.
#include <algorithm>
#include <type_traits>

#include "activation.h"
#include "layers.h"

namespace sgc {
namespace {

constexpr int kThreads = 256;
typedef float floatx4v __attribute__((ext_vector_type(4)));
typedef float floatx4_u __attribute__((ext_vector_type(4), aligned(4)));  // at any address

// Elements (i, j .. j + 7) of a rows x cols matrix, zeros outside it.
__device__ __forceinline__ void load8(const float* p, int64_t ld, int64_t i, int64_t j,
                                      int64_t rows, int64_t cols, float (&v)[8]) {
  const float* const at = p + i * ld + j;
  if (i < rows && j + 7 < cols) {
    const floatx4_u a = *reinterpret_cast<const floatx4_u*>(at);
    const floatx4_u b = *reinterpret_cast<const floatx4_u*>(at + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = a[e], v[e + 4] = b[e];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = i < rows && j + e < cols ? at[e] : 0.0f;
  }
}

// Four values from column j of a row of n, zeros past its end.
__device__ __forceinline__ floatx4v load4(const float* row, int64_t j, int64_t n) {
  if (j + 3 < n) return *reinterpret_cast<const floatx4_u*>(row + j);
  floatx4v v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = j + e < n ? row[j + e] : 0.0f;
  return v;
}

// The jobs of a launch; job b has blocks first[b] .. first[b + 1].
struct SplitArgs {
  SplitJob job[kSplitJobs];
  uint32_t first[kSplitJobs + 1];
  int count;
  float s;
  ColumnJoin join;
};

constexpr int kJoinLines = 32, kJoinGroups = kThreads / kJoinLines;

// Line j's sum or largest of `count` values, `stride` apart, in the first 32 threads
// (j < lines), every eighth value a thread.  `part`: a word per thread.
template <bool kMax>
__device__ __forceinline__ float join_line(const float* p, int count, int64_t stride,
                                           int64_t lines, int64_t j, float* part) {
  const int c = threadIdx.x % kJoinLines, q = threadIdx.x / kJoinLines;
  auto add = [](float x, float y) { return kMax ? __builtin_fmaxf(x, y) : x + y; };
  float s = 0.0f;
  if (j < lines) {
#pragma unroll 4
    for (int n = q; n < count; n += kJoinGroups) s = add(s, p[n * stride + j]);
  }
  part[q * kJoinLines + c] = s;
  __syncthreads();
  if (q == 0) {
#pragma unroll
    for (int n = 1; n < kJoinGroups; ++n) s = add(s, part[n * kJoinLines + c]);
  }
  return s;
}

__device__ __forceinline__ int shift_of(float top, int target) {
  return prescale_shift(__builtin_bit_cast(uint32_t, top), target);
}

// dbias of 32 columns.
__device__ void join_sums(const ColumnJoin& g, uint32_t block, float* part) {
  const int64_t j = static_cast<int64_t>(block) * kJoinLines + threadIdx.x % kJoinLines;
  const float s = join_line<false>(g.sums, g.slabs, g.N, g.N, j, part);
  if (threadIdx.x < kJoinLines && j < g.N) g.dbias[j] = s;
}

// The shifts of 32 rows or columns.
__device__ void join_shifts(const float* top, int count, int64_t stride, int64_t lines,
                            int target, int* shift, uint32_t block, float* part) {
  const int64_t j = static_cast<int64_t>(block) * kJoinLines + threadIdx.x % kJoinLines;
  const float m = join_line<true>(top, count, stride, lines, j, part);
  if (threadIdx.x < kJoinLines && j < lines) shift[j] = shift_of(m, target);
}

constexpr int kTileRows = 32, kTileCols = 128;
constexpr int kPitch = kTileRows / 2 + 4;  // words per column in LDS; 16-byte aligned

// A 32 x 128 tile of one matrix: thread t holds rows 2 (t / 16) and the next, 8
// columns from 8 (t % 16).  As row planes those are two 16-byte chunks of a tile
// row each.  As column planes the pairs of rows go to LDS as words, a column's
// side by side, and thread t writes chunk t of each of the tile's two slices.
// lines_of(): the shifts of this thread's two rows and eight columns, asked for once
// the tile's loads are on their way.  HBM bounds it: the gradient of 8192 x 4096 x 4096
// (dY times act'(Z) both ways, X and W) 150 us, 0.94 GB.
typedef int intx2 __attribute__((ext_vector_type(2)));
typedef int intx8 __attribute__((ext_vector_type(8)));
struct Shifts {
  intx2 row;
  intx8 col;
};
template <typename F>
__device__ __forceinline__ void split_tile(const SplitArgs& a, const SplitJob& g, uint32_t block,
                                           uint32_t* ph, uint32_t* pl, F lines_of) {
  const int t = threadIdx.x;
  const uint32_t strips = static_cast<uint32_t>((g.cols + kTileCols - 1) / kTileCols);
  const int64_t tr = block / strips, tc = block - static_cast<uint32_t>(tr) * strips;
  const int64_t i = tr * kTileRows + 2 * (t >> 4), j = tc * kTileCols + 8 * (t & 15);
  float v[2][8], z[2][8];
#pragma unroll
  for (int u = 0; u < 2; ++u) load8(g.s, g.ld, i + u, j, g.rows, g.cols, v[u]);
  if (g.z) {
#pragma unroll
    for (int u = 0; u < 2; ++u) load8(g.z, g.ldz, i + u, j, g.rows, g.cols, z[u]);
  }
  const bool scaled = g.row_shift || g.col_shift;
  Shifts lines;
  if (scaled) lines = lines_of(tr, tc);
  if (g.z) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[u][e] *= activate_grad(g.activation, z[u][e]);
  }
  const int64_t kp_row = (g.cols + kKPad - 1) / kKPad * kKPad;
  const int64_t kp_col = (g.rows + kKPad - 1) / kKPad * kKPad;
  bool big = false;
  auto too_big = [&](uint32_t h) {
    typedef _Float16 half2 __attribute__((ext_vector_type(2)));
    const half2 x = __builtin_bit_cast(half2, h);
    big |= __builtin_fabsf(static_cast<float>(x[0])) * a.s > 65504.0f;
    big |= __builtin_fabsf(static_cast<float>(x[1])) * a.s > 65504.0f;
  };
  // A pre-scaled operand's finite entries stay below the limit, and its infinities
  // belong in the result: no flag, whatever its words held (an earlier replay of a
  // captured call has the same stamp), as the GEMM has no fallback to run for it.
  auto flag = [&](uint32_t* range, uint32_t stamp) {
    if (big && !scaled) range[kWordBOverflow] = stamp;
    if (t == 0 && scaled) range[kWordBOverflow] = 0;  // no stamp is 0
    if (t == 0) range[kWordBStamp] = stamp;
  };
  if (g.row_hi && j < kp_row) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        w[e] = g.row_shift ? __builtin_ldexpf(v[u][e], lines.row[u]) : v[u][e];
      u32x4 hv, lv;
      split8(w, a.s, hv, lv);
      if (g.row_range) too_big(hv[0]), too_big(hv[1]), too_big(hv[2]), too_big(hv[3]);
      const int64_t at = tiled_index(i + u, j, kp_row);
      store_chunk(g.row_hi + at, hv);
      store_chunk(g.row_lo + at, lv);
    }
  }
  if (g.row_range) flag(g.row_range, g.row_stamp);
  if (!g.col_hi) return;
  big = false;
  const int cl = 8 * (t & 15), rp = t >> 4;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (g.col_shift) {
      v[0][e] = __builtin_ldexpf(v[0][e], lines.col[e]);
      v[1][e] = __builtin_ldexpf(v[1][e], lines.col[e]);
    }
    uint16_t h0, l0, h1, l1;
    split_value(v[0][e], a.s, h0, l0);
    split_value(v[1][e], a.s, h1, l1);
    const uint32_t h = static_cast<uint32_t>(h0) | (static_cast<uint32_t>(h1) << 16);
    if (g.col_range) too_big(h);
    ph[(cl + e) * kPitch + rp] = h;
    pl[(cl + e) * kPitch + rp] = static_cast<uint32_t>(l0) | (static_cast<uint32_t>(l1) << 16);
  }
  if (g.col_range) flag(g.col_range, g.col_stamp);
  __syncthreads();
  const int r = t >> 1, c = (t & 1) ^ tile_swizzle(r);
#pragma unroll
  for (int sl = 0; sl < kTileRows / kSlice; ++sl) {
    const int64_t at = (tc * (kp_col / kSlice) + tr * (kTileRows / kSlice) + sl) * kTileHalves + t * 8;
    store_chunk(g.col_hi + at, *reinterpret_cast<const u32x4*>(ph + r * kPitch + sl * 8 + c * 4));
    store_chunk(g.col_lo + at, *reinterpret_cast<const u32x4*>(pl + r * kPitch + sl * 8 + c * 4));
  }
}

__global__ __launch_bounds__(kThreads) void split_jobs_kernel(SplitArgs a) {
  __shared__ __align__(16) uint32_t ph[kTileCols * kPitch];
  __shared__ __align__(16) uint32_t pl[kTileCols * kPitch];
  for (uint32_t b = blockIdx.x; b < a.first[a.count]; b += gridDim.x) {
    int n = 0;
    while (n + 1 < a.count && b >= a.first[n + 1]) ++n;
    const SplitJob& g = a.job[n];
    split_tile(a, g, b - a.first[n], ph, pl, [&](int64_t tr, int64_t tc) {
      // Past the end the shifts are anything, and the values that take them 0.
      Shifts s{};
      if (g.row_shift)
        s.row = *reinterpret_cast<const intx2*>(g.row_shift + tr * kTileRows +
                                                2 * (threadIdx.x >> 4));
      if (g.col_shift)
        s.col = *reinterpret_cast<const intx8*>(g.col_shift + tc * kTileCols +
                                                8 * (threadIdx.x & 15));
      return s;
    });
    __syncthreads();  // the tile's LDS words are read before the next's are written
  }
}

// A tile's shifts from what launch_columns left.  Both lines' largest magnitudes are
// joined in LDS: 32 rows by eight threads each over the strips, 128 columns by eight
// threads to four of them over the slabs.
__device__ __forceinline__ Shifts join_tile(const ColumnJoin& g, int64_t tr, int64_t tc,
                                            float* col_part, float* row_part) {
  __shared__ __align__(32) int rows[kTileRows], cols[kTileCols];
  static_assert(kTileRows == kJoinLines && kTileCols == 4 * kJoinLines &&
                kTileRows + kTileCols <= kThreads, "threads to a line");
  const int t = threadIdx.x, l = t % kJoinLines, q = t / kJoinLines;
  const int64_t i0 = tr * kTileRows, j0 = tc * kTileCols;
  float m[4] = {0.0f, 0.0f, 0.0f, 0.0f}, top = 0.0f;
  if (g.col_shift) {
    const int64_t stride = (g.N + kColumnStrip - 1) / kColumnStrip * kColumnStrip;
#pragma unroll 8
    for (int n = q; n < g.slabs; n += kJoinGroups) {
      const floatx4v x = *reinterpret_cast<const floatx4v*>(g.col_top + n * stride + j0 + 4 * l);
#pragma unroll
      for (int e = 0; e < 4; ++e) m[e] = __builtin_fmaxf(m[e], x[e]);
    }
  }
  if (g.row_shift && i0 + l < g.M) {
#pragma unroll 8
    for (int n = q; n < g.pieces; n += kJoinGroups)
      top = __builtin_fmaxf(top, g.row_top[n * g.M + i0 + l]);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) col_part[q * kTileCols + 4 * l + e] = m[e];
  row_part[q * kTileRows + l] = top;
  __syncthreads();
  if (t < kTileCols) {
    float c = col_part[t];
#pragma unroll
    for (int n = 1; n < kJoinGroups; ++n) c = __builtin_fmaxf(c, col_part[n * kTileCols + t]);
    cols[t] = shift_of(c, g.col_target);
    if (g.col_shift && tr == 0 && j0 + t < g.N) g.col_shift[j0 + t] = cols[t];
  } else if (t < kTileCols + kTileRows) {
    const int k = t - kTileCols;
    float r = row_part[k];
#pragma unroll
    for (int n = 1; n < kJoinGroups; ++n) r = __builtin_fmaxf(r, row_part[n * kTileRows + k]);
    rows[k] = shift_of(r, g.row_target);
    if (g.row_shift && tc == 0 && i0 + k < g.M) g.row_shift[i0 + k] = rows[k];
  }
  __syncthreads();
  return {*reinterpret_cast<const intx2*>(rows + 2 * (t >> 4)),
          *reinterpret_cast<const intx8*>(cols + 8 * (t & 15))};
}

// With the join: a tile a workgroup, then the workgroups of dbias.
__global__ __launch_bounds__(kThreads) void split_join_kernel(SplitArgs a) {
  __shared__ __align__(16) uint32_t ph[kTileCols * kPitch];
  __shared__ __align__(16) uint32_t pl[kTileCols * kPitch];
  const uint32_t b = blockIdx.x;
  if (b >= a.first[a.count]) {
    join_sums(a.join, b - a.first[a.count], reinterpret_cast<float*>(ph));
    return;
  }
  int n = 0;
  while (n + 1 < a.count && b >= a.first[n + 1]) ++n;
  split_tile(a, a.job[n], b - a.first[n], ph, pl, [&](int64_t tr, int64_t tc) {
    return join_tile(a.join, tr, tc, reinterpret_cast<float*>(ph), reinterpret_cast<float*>(pl));
  });
}

// Rows that a thread has in flight.
constexpr int kColumnRows = 4;

// Largest of 16 lanes, by rotations.
__device__ __forceinline__ float quarter_max(float v) {
  auto step = [&](auto control) {
    const int o = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v),
                                              decltype(control)::value, 0xf, 0xf, true);
    v = __builtin_fmaxf(v, __builtin_bit_cast(float, o));
  };
  step(std::integral_constant<int, 0x121>{});  // row_ror:1
  step(std::integral_constant<int, 0x122>{});
  step(std::integral_constant<int, 0x124>{});
  step(std::integral_constant<int, 0x128>{});
  return v;
}

// 128 columns of a slab of rows: thread t has columns 4 (t % 32) .. + 3 of every
// eighth row, so that 16 lanes also find the largest magnitude of half of its strip.
// 8192 x 4096 with Z: 46 us, 5.8 TB/s.
__global__ __launch_bounds__(kThreads) void columns_kernel(ColumnArgs a, int64_t slab_rows) {
  __shared__ float sums[kThreads / 32][kColumnStrip], tops[kThreads / 32][kColumnStrip];
  const int t = threadIdx.x;
  const int64_t j = static_cast<int64_t>(blockIdx.x) * kColumnStrip + 4 * (t & 31);
  const int64_t i0 = blockIdx.y * slab_rows, i1 = min(a.M, i0 + slab_rows);
  float s[4] = {0.0f, 0.0f, 0.0f, 0.0f}, top[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  constexpr int kStride = kThreads / 32;
  // Rows i, i + 8, ... (kU) of a whole strip or (not kFull) of the last: all lanes of a
  // row take every step together.
  auto rows = [&](int64_t i, auto count, auto whole) {
    constexpr int kU = decltype(count)::value;
    constexpr bool kFull = decltype(whole)::value;
    auto load = [&](const float* row) {
      if constexpr (kFull) return floatx4v(*reinterpret_cast<const floatx4_u*>(row + j));
      else return load4(row, j, a.N);
    };
    floatx4v d[kU], z[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) d[u] = load(a.dy + (i + u * kStride) * a.lddy);
    if (a.z) {
#pragma unroll
      for (int u = 0; u < kU; ++u) z[u] = load(a.z + (i + u * kStride) * a.ldz);
      multiply_grad(a.activation, d, z);
    }
    if (a.d) {
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        float* const at = a.d + (i + u * kStride) * a.N + j;
        if (kFull || j + 3 < a.N) {
          *reinterpret_cast<floatx4_u*>(at) = d[u];
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (j + e < a.N) at[e] = d[u][e];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      float b[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[e] += d[u][e];
        b[e] = __builtin_fabsf(d[u][e]);
        b[e] = b[e] <= 3.4028235e38f ? b[e] : 0.0f;
        top[e] = __builtin_fmaxf(top[e], b[e]);
      }
      if (a.row_top) {
        const float m = quarter_max(__builtin_fmaxf(__builtin_fmaxf(b[0], b[1]),
                                                    __builtin_fmaxf(b[2], b[3])));
        if ((t & 15) == 0)
          a.row_top[(2 * blockIdx.x + (t >> 4 & 1)) * a.M + i + u * kStride] = m;
      }
    }
  };
  auto slab = [&](auto whole) {
    int64_t i = i0 + (t >> 5);
    for (; i + (kColumnRows - 1) * kStride < i1; i += kColumnRows * kStride)
      rows(i, std::integral_constant<int, kColumnRows>{}, whole);
    for (; i < i1; i += kStride) rows(i, std::integral_constant<int, 1>{}, whole);
  };
  if ((blockIdx.x + 1) * static_cast<int64_t>(kColumnStrip) <= a.N)
    slab(std::true_type{});
  else
    slab(std::false_type{});
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    sums[t >> 5][4 * (t & 31) + e] = s[e];
    tops[t >> 5][4 * (t & 31) + e] = top[e];
  }
  __syncthreads();
  const int64_t col = static_cast<int64_t>(blockIdx.x) * kColumnStrip + t;
  if (t >= kColumnStrip) return;
  float sum = 0.0f, most = 0.0f;
#pragma unroll
  for (int g = 0; g < kThreads / 32; ++g) {
    sum += sums[g][t];
    most = __builtin_fmaxf(most, tops[g][t]);
  }
  if (col < a.N) a.sums[blockIdx.y * a.N + col] = sum;
  if (a.col_top)
    a.col_top[blockIdx.y * (static_cast<int64_t>(gridDim.x) * kColumnStrip) + col] = most;
}

// The join alone, 32 columns or rows a workgroup: dbias, the columns' shifts, the rows'.
__global__ __launch_bounds__(kThreads) void columns_join_kernel(ColumnJoin g, uint32_t sums,
                                                                uint32_t cols) {
  __shared__ float part[kThreads];
  if (blockIdx.x < sums)
    join_sums(g, blockIdx.x, part);
  else if (blockIdx.x < sums + cols)
    join_shifts(g.col_top, g.slabs, (g.N + kColumnStrip - 1) / kColumnStrip * kColumnStrip, g.N,
                g.col_target, g.col_shift, blockIdx.x - sums, part);
  else
    join_shifts(g.row_top, g.pieces, g.M, g.M, g.row_target, g.row_shift,
                blockIdx.x - sums - cols, part);
}

// The epilogue of a product without terms: Z = bias.
__global__ __launch_bounds__(kThreads) void epilogue_kernel(Epilogue e, int64_t M, int64_t N,
                                                            float* Y, int64_t ldy) {
  const int64_t j = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (j >= N) return;
  const float z = e.bias ? e.bias[j] : 0.0f, y = activate(e.activation, z);
  for (int64_t i = blockIdx.y; i < M; i += gridDim.y) {
    if (e.z) e.z[i * e.ldz + j] = z;
    Y[i * ldy + j] = e.r ? y + e.r[i * e.ldr + j] : y;
  }
}

}  // namespace

namespace {

// Tiles of a job.  Rows up to a multiple of 64: the padding of k in column planes.
int64_t job_blocks(const SplitJob& j) {
  return round_up(j.rows, kKPad) / kTileRows * ((j.cols + kTileCols - 1) / kTileCols);
}

unsigned join_blocks(const void* wanted, int64_t lines) {
  return wanted ? static_cast<unsigned>((lines + kJoinLines - 1) / kJoinLines) : 0u;
}

}  // namespace

int64_t split_jobs_blocks(const SplitJob* jobs, int count) {
  int64_t blocks = 0;
  for (int n = 0; n < count; ++n) blocks += job_blocks(jobs[n]);
  return blocks;
}

hipError_t launch_split_jobs(const SplitJob* jobs, int count, float scale, hipStream_t stream,
                             const ColumnJoin* join) {
  SplitArgs a{};
  a.s = scale;
  a.count = count;
  int64_t blocks = 0;
  for (int n = 0; n < count; ++n) {
    a.job[n] = jobs[n];
    a.first[n] = static_cast<uint32_t>(blocks);
    blocks += job_blocks(jobs[n]);
    if (blocks > UINT32_MAX) return hipErrorInvalidValue;
  }
  a.first[count] = static_cast<uint32_t>(blocks);
  if (blocks == 0) return hipSuccess;
  if (join) {
    a.join = *join;
    hipLaunchKernelGGL(split_join_kernel, dim3(a.first[count] + join_blocks(join->dbias, join->N)),
                       dim3(kThreads), 0, stream, a);
    return hipGetLastError();
  }
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(blocks, int64_t{1} << 22)));
  hipLaunchKernelGGL(split_jobs_kernel, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

int64_t column_strips(int64_t N) { return (N + kColumnStrip - 1) / kColumnStrip; }

int64_t column_slabs(int64_t M, int64_t N) {
  return std::max<int64_t>(1, std::min<int64_t>((M + 31) / 32, 1024 / column_strips(N)));
}

hipError_t launch_columns(const ColumnArgs& a, hipStream_t stream) {
  const int64_t slabs = column_slabs(a.M, a.N);
  hipLaunchKernelGGL(columns_kernel, dim3(static_cast<unsigned>(column_strips(a.N)),
                                          static_cast<unsigned>(slabs)),
                     dim3(kThreads), 0, stream, a, (a.M + slabs - 1) / slabs);
  return hipGetLastError();
}

hipError_t launch_columns_join(const ColumnJoin& j, hipStream_t stream) {
  const unsigned sums = join_blocks(j.dbias, j.N), cols = join_blocks(j.col_shift, j.N);
  const unsigned rows = join_blocks(j.row_shift, j.M);
  if (sums + cols + rows == 0) return hipSuccess;
  hipLaunchKernelGGL(columns_join_kernel, dim3(sums + cols + rows), dim3(kThreads), 0, stream, j,
                     sums, cols);
  return hipGetLastError();
}

hipError_t launch_epilogue(const Epilogue& e, int64_t M, int64_t N, float* Y, int64_t ldy,
                           hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>((N + kThreads - 1) / kThreads),
                  static_cast<unsigned>(std::min<int64_t>(M, 65535)));
  hipLaunchKernelGGL(epilogue_kernel, grid, dim3(kThreads), 0, stream, e, M, N, Y, ldy);
  return hipGetLastError();
}

}  // namespace sgc
