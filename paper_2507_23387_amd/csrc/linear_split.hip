// What a linear layer's products need around them (gfx950): the split of its
// operands into planes in either direction, the gradient D = dY act'(Z) with its
// column sums and largest magnitude, and the epilogue.
#include <algorithm>

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

// The jobs of a launch; job b has blocks first[b] .. first[b + 1].
struct SplitArgs {
  SplitJob job[kSplitJobs];
  uint32_t first[kSplitJobs + 1];
  int count;
  float s;
  ColumnJoin join;
};

constexpr int kJoinCols = 32, kJoinGroups = kThreads / kJoinCols;

// The largest of the slabs' magnitudes, in every thread.  `lds`: a word per wave.
__device__ uint32_t join_top(const ColumnJoin& g, float* lds) {
  const int t = threadIdx.x;
  float m = 0.0f;
#pragma unroll 4
  for (int n = t; n < g.tops; n += kThreads) m = __builtin_fmaxf(m, g.top[n]);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) m = __builtin_fmaxf(m, __shfl_xor(m, off));
  if ((t & 63) == 0) lds[t >> 6] = m;
  __syncthreads();
  m = __builtin_fmaxf(__builtin_fmaxf(lds[0], lds[1]), __builtin_fmaxf(lds[2], lds[3]));
  return __builtin_bit_cast(uint32_t, m);
}

// dbias of 32 columns, every eighth slab a thread.  `part`: a word per thread.
__device__ void join_columns(const ColumnJoin& g, uint32_t block, float* part) {
  const int c = threadIdx.x % kJoinCols, q = threadIdx.x / kJoinCols;
  const int64_t j = static_cast<int64_t>(block) * kJoinCols + c;
  float s = 0.0f;
  if (j < g.N) {
#pragma unroll 4
    for (int n = q; n < g.slabs; n += kJoinGroups) s += g.sums[n * g.N + j];
  }
  part[q * kJoinCols + c] = s;
  __syncthreads();
  if (q != 0 || j >= g.N) return;
#pragma unroll
  for (int n = 1; n < kJoinGroups; ++n) s += part[n * kJoinCols + c];
  g.dbias[j] = s;
}

constexpr int kTileRows = 32, kTileCols = 128;
constexpr int kPitch = kTileRows / 2 + 4;  // words per column in LDS; 16-byte aligned

// A 32 x 128 tile of one matrix: thread t holds rows 2 (t / 16) and the next, 8
// columns from 8 (t % 16).  As row planes those are two 16-byte chunks of a tile
// row each.  As column planes the pairs of rows go to LDS as words, a column's
// side by side, and thread t writes chunk t of each of the tile's two slices.
// max_bits(): the bits of the magnitude that a job is scaled by, asked for once the
// tile's loads are on their way.  HBM bounds it: the gradient of 8192 x 4096 x 4096 (dY
// times act'(Z) both ways, X and W) 150 us, 0.94 GB.
template <typename F>
__device__ __forceinline__ void split_tile(const SplitArgs& a, const SplitJob& g, uint32_t block,
                                           uint32_t* ph, uint32_t* pl, F max_bits_of) {
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
  const uint32_t max_bits = g.max_bits ? max_bits_of() : 0;
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
    if (big && !g.max_bits) range[kWordBOverflow] = stamp;
    if (t == 0 && g.max_bits) range[kWordBOverflow] = 0;  // no stamp is 0
    if (t == 0) range[kWordBStamp] = stamp;
  };
  if (g.row_hi && j < kp_row) {
    const int shift = g.max_bits ? prescale_shift(max_bits, g.row_target) : 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = shift ? __builtin_ldexpf(v[u][e], shift) : v[u][e];
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
  const int shift = g.max_bits ? prescale_shift(max_bits, g.col_target) : 0;
  const int cl = 8 * (t & 15), rp = t >> 4;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    uint16_t h0, l0, h1, l1;
    split_value(shift ? __builtin_ldexpf(v[0][e], shift) : v[0][e], a.s, h0, l0);
    split_value(shift ? __builtin_ldexpf(v[1][e], shift) : v[1][e], a.s, h1, l1);
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
    split_tile(a, g, b - a.first[n], ph, pl, [&] { return *g.max_bits; });
    __syncthreads();  // the tile's LDS words are read before the next's are written
  }
}

// With the join: a tile a workgroup, then the join's workgroups.
__global__ __launch_bounds__(kThreads) void split_join_kernel(SplitArgs a) {
  __shared__ __align__(16) uint32_t ph[kTileCols * kPitch];
  __shared__ __align__(16) uint32_t pl[kTileCols * kPitch];
  const uint32_t b = blockIdx.x;
  if (b >= a.first[a.count]) {
    join_columns(a.join, b - a.first[a.count], reinterpret_cast<float*>(ph));
    return;
  }
  int n = 0;
  while (n + 1 < a.count && b >= a.first[n + 1]) ++n;
  const SplitJob& g = a.job[n];
  split_tile(a, g, b - a.first[n], ph, pl, [&] {
    const uint32_t bits = join_top(a.join, reinterpret_cast<float*>(pl));
    if (b == a.first[n] && threadIdx.x == 0) *a.join.max_bits = bits;
    __syncthreads();  // pl is read before the tile is written
    return bits;
  });
}

// Rows that a thread has in flight.
constexpr int kColumnRows = 4;

// Sums of 128 columns over a slab of rows: thread t has columns 4 (t % 32) .. + 3
// of every eighth row.  8192 x 4096 with Z: 44 us, 6.1 TB/s.
__global__ __launch_bounds__(kThreads) void columns_kernel(ColumnArgs a, int64_t slab_rows) {
  __shared__ float part[kThreads / 32][kColumnStrip];
  __shared__ float top[kThreads / 64];
  const int t = threadIdx.x;
  const int64_t j = static_cast<int64_t>(blockIdx.x) * kColumnStrip + 4 * (t & 31);
  const int64_t i0 = blockIdx.y * slab_rows, i1 = min(a.M, i0 + slab_rows);
  float s[4] = {0.0f, 0.0f, 0.0f, 0.0f}, m = 0.0f;
  auto add = [&](const float (&d)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[e] += d[e];
      const float b = __builtin_fabsf(d[e]);
      if (b <= 3.4028235e38f) m = __builtin_fmaxf(m, b);
    }
  };
  constexpr int kStride = kThreads / 32;
  int64_t i = i0 + (t >> 5);
  if (j + 3 < a.N) {
    for (; i + (kColumnRows - 1) * kStride < i1; i += kColumnRows * kStride) {
      floatx4v d[kColumnRows], z[kColumnRows];
#pragma unroll
      for (int u = 0; u < kColumnRows; ++u)
        d[u] = *reinterpret_cast<const floatx4_u*>(a.dy + (i + u * kStride) * a.lddy + j);
      if (a.z) {
#pragma unroll
        for (int u = 0; u < kColumnRows; ++u)
          z[u] = *reinterpret_cast<const floatx4_u*>(a.z + (i + u * kStride) * a.ldz + j);
        multiply_grad(a.activation, d, z);
      }
      if (a.d) {
#pragma unroll
        for (int u = 0; u < kColumnRows; ++u)
          *reinterpret_cast<floatx4_u*>(a.d + (i + u * kStride) * a.N + j) = d[u];
      }
#pragma unroll
      for (int u = 0; u < kColumnRows; ++u) add({d[u][0], d[u][1], d[u][2], d[u][3]});
    }
  }
  for (; i < i1; i += kStride) {
    float d[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      d[e] = j + e < a.N ? a.dy[i * a.lddy + j + e] : 0.0f;
      if (a.z && j + e < a.N) d[e] *= activate_grad(a.activation, a.z[i * a.ldz + j + e]);
      if (a.d && j + e < a.N) a.d[i * a.N + j + e] = d[e];
    }
    add(d);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) part[t >> 5][4 * (t & 31) + e] = s[e];
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) m = __builtin_fmaxf(m, __shfl_xor(m, off));
  if ((t & 63) == 0) top[t >> 6] = m;
  __syncthreads();
  const int64_t col = static_cast<int64_t>(blockIdx.x) * kColumnStrip + t;
  if (t < kColumnStrip && col < a.N) {
    float sum = 0.0f;
#pragma unroll
    for (int g = 0; g < kThreads / 32; ++g) sum += part[g][t];
    a.partial[blockIdx.y * a.N + col] = sum;
  }
  if (t == 0)
    a.partial[gridDim.y * a.N + blockIdx.y * gridDim.x + blockIdx.x] = __builtin_fmaxf(__builtin_fmaxf(top[0], top[1]),
                                            __builtin_fmaxf(top[2], top[3]));
}

// The join alone: every workgroup but the last has 32 columns.
__global__ __launch_bounds__(kThreads) void columns_join_kernel(ColumnJoin g) {
  __shared__ float part[kThreads];
  if (blockIdx.x < gridDim.x - 1) {
    join_columns(g, blockIdx.x, part);
  } else {
    const uint32_t bits = join_top(g, part);
    if (threadIdx.x == 0) *g.max_bits = bits;
  }
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

unsigned join_blocks(const ColumnJoin& j) {
  return j.dbias ? static_cast<unsigned>((j.N + kJoinCols - 1) / kJoinCols) : 0u;
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
    hipLaunchKernelGGL(split_join_kernel, dim3(a.first[count] + join_blocks(*join)),
                       dim3(kThreads), 0, stream, a);
    return hipGetLastError();
  }
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(blocks, int64_t{1} << 22)));
  hipLaunchKernelGGL(split_jobs_kernel, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

int64_t column_slabs(int64_t M, int64_t N) {
  const int64_t strips = (N + kColumnStrip - 1) / kColumnStrip;
  return std::max<int64_t>(1, std::min<int64_t>((M + 31) / 32, 1024 / strips));
}

hipError_t launch_columns(const ColumnArgs& a, hipStream_t stream) {
  const int64_t strips = (a.N + kColumnStrip - 1) / kColumnStrip;
  const int64_t slabs = column_slabs(a.M, a.N);
  hipLaunchKernelGGL(columns_kernel, dim3(static_cast<unsigned>(strips), static_cast<unsigned>(slabs)),
                     dim3(kThreads), 0, stream, a, (a.M + slabs - 1) / slabs);
  return hipGetLastError();
}

ColumnJoin column_join(const ColumnArgs& a) {
  const int64_t slabs = column_slabs(a.M, a.N), strips = (a.N + kColumnStrip - 1) / kColumnStrip;
  return ColumnJoin{a.partial + slabs * a.N, static_cast<int>(slabs * strips), a.max_bits,
                    a.partial, static_cast<int>(slabs), a.N, a.dbias};
}

hipError_t launch_columns_join(const ColumnJoin& j, hipStream_t stream) {
  hipLaunchKernelGGL(columns_join_kernel, dim3(join_blocks(j) + 1), dim3(kThreads), 0, stream, j);
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
