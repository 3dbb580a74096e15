// The linear layer and its gradients: workspace, operands and launches.
#include <algorithm>
#include <cmath>

#include "layers.h"

namespace sgc {
namespace {

// One product's planes, carved from a workspace: a_rows x k and b_rows x k.
struct Carver {
  char* base;
  size_t used;
  template <typename T>
  T* take(int64_t count) {
    char* const at = base + used;
    used += static_cast<size_t>(round_up(count * static_cast<int64_t>(sizeof(T)), 256));
    return reinterpret_cast<T*>(at);
  }
};

Planes carve_planes(Carver& c, int64_t M, int64_t N, int64_t K) {
  Planes p{};
  p.Mp = round_up(M, kRowPad);
  p.Np = round_up(N, kRowPad);
  p.Kp = round_up(K, kKPad);
  p.range = c.take<uint32_t>(kFlagBytes / 4);
  p.a_hi = c.take<uint16_t>(p.Mp * p.Kp);
  p.a_lo = c.take<uint16_t>(p.Mp * p.Kp);
  p.b_hi = c.take<uint16_t>(p.Np * p.Kp);
  p.b_lo = c.take<uint16_t>(p.Np * p.Kp);
  return p;
}

SplitJob job_of(const float* s, int64_t ld, int64_t rows, int64_t cols) {
  SplitJob j{};
  j.s = s;
  j.ld = ld;
  j.rows = rows;
  j.cols = cols;
  return j;
}

// Adds planes to a job: the A or the B side of p, from its rows or its columns.
void to_planes(SplitJob& j, const Planes& p, bool side_b, bool columns) {
  uint16_t* const hi = side_b ? p.b_hi : p.a_hi;
  uint16_t* const lo = side_b ? p.b_lo : p.a_lo;
  if (columns) {
    j.col_hi = hi, j.col_lo = lo;
    if (side_b) j.col_range = p.range, j.col_stamp = next_stamp();
  } else {
    j.row_hi = hi, j.row_lo = lo;
    if (side_b) j.row_range = p.range, j.row_stamp = next_stamp();
  }
}

// Most tiles of a split that also joins what the pass over D left: each of D's tiles
// then joins its own lines' magnitudes, 2 us and more where they are many, instead of
// a launch between (us, so and with it: 256 x 1024 x 1024 27.9 and 28.9, 777 x 1003 x 530
// 30.8 and 32.7, 4096 x 256 x 256 39.8 and 41.6, 1024 x 1024 x 512 30.3 and 30.6; of more
// tiles 2048 x 1024 x 1024 56.1 and 55.4, 2048 x 2560 x 512 79.5 and 73.0).
constexpr int64_t kSplitJoinBlocks = 1024;

// Target exponents of a pre-scaled operand (api.hip's range_opts): as A, and as
// B, where the scaled kernels form s B_hi in FP16.
int target_a(float scale) { return std::min(14, 26 - std::ilogb(scale)); }
int target_b(float scale, int variant) {
  return variant == kTermwise || !scaled_kernel_ok(scale) ? target_a(scale)
                                                          : 14 - std::ilogb(scale);
}

}  // namespace

// Few rows: every 64 rows read W once more, as FP32, where the tiles read it,
// write its planes and read those for every 32 to 256 rows.  On N, K = 256 .. 8192,
// rows against tiles, us: 64 x 4096 x 4096 27 and 42, 128 x 4096 x 4096 38 and 51, 128
// x 8192 x 8192 120 and 185, 256 x 512 x 4096 17 and 26; 192 x 4096 x 4096 49 and 54,
// 256 x 2048 x 2048 23 and 28, but 256 x 4096 x 4096 59 and 58, 192 x 8192 x 4096 89 to
// 106 and 96, 384 x 2048 x 4096 45 to 52 and 45.
bool linear_by_rows(int64_t M, int64_t N) {
  return M <= 128 || (M <= 256 && M * N <= 800000);
}

// Few columns: the same with the sides exchanged, X read once as FP32 instead of
// its planes written and read too.  Against tiles, us: 16384 x 1 x 8192 94 and 304,
// 16384 x 64 x 2048 51 and 71, 300 x 128 x 8192 19 and 40, 16384 x 128 x 2048 76 and 82,
// 4000 x 128 x 512 19 and 18, 1000 x 256 x 2048 21 and 21, but 4000 x 192 x 2048 38 and
// 33.  (The bound on M keeps the grid below 2^32 threads.)
bool linear_by_columns(int64_t M, int64_t N) {
  return M <= (int64_t{1} << 25) && (N <= 128 || (N <= 256 && M * N <= 300000));
}

size_t linear_ws(int64_t M, int64_t N, int64_t K) {
  if (M == 0 || N == 0 || K == 0) return 0;
  if (linear_by_rows(M, N)) return linear_rows_ws(M, N, K);
  if (linear_by_columns(M, N)) return linear_rows_ws(N, M, K);
  Carver c{nullptr, 0};
  (void)carve_planes(c, M, N, K);
  return c.used;
}

hipError_t launch_linear(const LinearArgs& a, void* ws, hipStream_t stream) {
  if (a.K == 0) return launch_epilogue(a.e, a.M, a.N, a.y, a.ldy, stream);
  if (linear_by_rows(a.M, a.N)) return launch_linear_rows(a, nullptr, ws, stream);
  if (linear_by_columns(a.M, a.N)) return launch_linear_columns(a, ws, stream);
  Carver c{static_cast<char*>(ws), 0};
  const Planes p = carve_planes(c, a.M, a.N, a.K);
  SplitJob jobs[2] = {a.transpose_w ? job_of(a.w, a.ldw, a.N, a.K)
                                    : job_of(a.w, a.ldw, a.K, a.N),
                      job_of(a.x, a.ldx, a.M, a.K)};
  to_planes(jobs[0], p, true, !a.transpose_w);
  to_planes(jobs[1], p, false, false);
  const bool x_in_gemm = splits_a_in_gemm(a.M, a.N, a.x, a.ldx, a.K, a.scale, a.variant);
  const hipError_t err = launch_split_jobs(jobs, x_in_gemm ? 1 : 2, a.scale, stream);
  if (err != hipSuccess) return err;
  if (x_in_gemm)
    return launch_gemm_fused_a_epilogue(p, a.M, a.N, a.K, a.x, a.ldx, a.y, a.ldy, a.scale,
                                        a.variant, a.e, stream);
  return launch_gemm_epilogue(p, a.M, a.N, a.y, a.ldy, a.scale, a.variant, a.e, false,
                              stream);
}

namespace {

// Whether dX = D W^T (M x K, k over N) goes by rows.  D is then written as FP32 by
// the kernel that sums its columns, where an activation makes it other than dY.  A
// small W is split with the rest instead, and both products take one launch (us,
// rows against that: 64 rows, 1024 x 1024 30 and 25, 1024 x 2048 30 and 30, 2048 x
// 2048 32 and 39, 4096 x 4096 58 and 75; 256 rows 4096 x 4096 122 and 104).  A long k
// for few tiles takes longer still, while rows share it (N x K, 1 and 128 rows: 2048 x
// 512 25 and 27 against 27 and 29, 3000 x 128 25 and 27 against 23 and 25, 4096 x 128 28
// against 32, 8192 x 64 28 and 31 against 45 and 48).
bool grad_by_rows(int64_t M, int64_t N, int64_t K) {
  return M <= 128 && (N * K >= 1500000 || static_cast<double>(N) * N * K >= 1.6e9);
}

// Whether dW = X^T D is formed in FP32 from few rows, where dX needs no planes of D
// either.
bool grad_outer(int64_t M, int64_t N, int64_t K) {
  return M <= kOuterRows && grad_by_rows(M, N, K);
}

struct GradWorkspace {
  float *row_top, *col_top, *sums;  // launch_columns' arrays
  int *row_shift, *col_shift;
  void* rows;  // launch_linear_rows' workspace
  float* d;    // M x N, by rows
  Planes dx, dw;
  size_t bytes;
};

GradWorkspace carve_grad(void* ws, int64_t M, int64_t N, int64_t K, bool transpose_w) {
  Carver c{static_cast<char*>(ws), 0};
  GradWorkspace g{};
  const int64_t slabs = column_slabs(M, N);
  g.row_top = c.take<float>(row_pieces(N) * M);
  g.col_top = c.take<float>(slabs * round_up(N, kColumnStrip));
  g.sums = c.take<float>(slabs * N);
  g.row_shift = c.take<int>(round_up(M, kKPad));
  g.col_shift = c.take<int>(round_up(N, kColumnStrip));
  if (K > 0) {
    if (grad_by_rows(M, N, K)) {
      g.rows = c.take<char>(static_cast<int64_t>(linear_rows_ws(M, K, N)));
      g.d = c.take<float>(M * N);
    } else {
      g.dx = carve_planes(c, M, K, N);
    }
    if (!grad_outer(M, N, K))
      g.dw = transpose_w ? carve_planes(c, N, K, M) : carve_planes(c, K, N, M);
  }
  g.bytes = c.used;
  return g;
}

}  // namespace

size_t linear_grad_ws(int64_t M, int64_t N, int64_t K) {
  if (M == 0 || N == 0) return 0;
  return carve_grad(nullptr, M, N, K, false).bytes;
}

hipError_t launch_linear_grad(const LinearGradArgs& a, void* ws, hipStream_t stream) {
  hipError_t err = hipSuccess;
  const int64_t dw_rows = a.transpose_w ? a.N : a.K, dw_cols = a.transpose_w ? a.K : a.N;
  if (a.M == 0 || a.N == 0) {
    // No rows: the sums are empty.  No columns: dX = 0.
    if (a.dx) err = launch_zero(a.M, a.K, a.dx, a.lddx, stream);
    if (err == hipSuccess && a.dw) err = launch_zero(dw_rows, dw_cols, a.dw, a.lddw, stream);
    if (err == hipSuccess && a.dbias) err = launch_zero(1, a.N, a.dbias, a.N, stream);
    return err;
  }
  const GradWorkspace g = carve_grad(ws, a.M, a.N, a.K, a.transpose_w);
  const bool dx = a.dx && a.K > 0, outer = a.dw && a.K > 0 && grad_outer(a.M, a.N, a.K);
  const bool dw = a.dw && a.K > 0 && !outer;
  const bool dx_rows = dx && grad_by_rows(a.M, a.N, a.K);
  // dX is scaled by rows, dW by columns: each of their entries sums one line of D, so
  // that a line far below the others keeps its digits.
  const ColumnArgs cols{a.M, a.N, a.dy, a.lddy, a.z, a.ldz, a.activation,
                        dx ? g.row_top : nullptr, dw ? g.col_top : nullptr, g.sums,
                        dx_rows && a.z ? g.d : nullptr};
  ColumnJoin join{};
  join.M = a.M, join.N = a.N;
  join.pieces = static_cast<int>(row_pieces(a.N));
  join.slabs = static_cast<int>(column_slabs(a.M, a.N));
  join.row_top = g.row_top, join.col_top = g.col_top, join.sums = g.sums;
  join.row_target = target_a(a.scale);
  join.col_target = a.transpose_w ? target_a(a.scale) : target_b(a.scale, a.variant);
  join.row_shift = dx ? g.row_shift : nullptr;
  join.col_shift = dw ? g.col_shift : nullptr;
  join.dbias = a.dbias;

  SplitJob jobs[kSplitJobs];
  int count = 0;
  SplitJob d = cols.d ? job_of(cols.d, a.N, a.M, a.N) : job_of(a.dy, a.lddy, a.M, a.N);
  if (!cols.d) d.z = a.z, d.ldz = a.ldz, d.activation = a.activation;
  // In dW, D's columns are the result's columns, or with N x K weights its rows.
  const Unscale ex{g.row_shift, false}, ew{g.col_shift, !a.transpose_w};
  if (dx && !dx_rows) {
    // dX = D W^T: D's rows and W's K rows, k over N.
    d.row_shift = g.row_shift;
    to_planes(d, g.dx, false, false);
    jobs[count] = a.transpose_w ? job_of(a.w, a.ldw, a.N, a.K) : job_of(a.w, a.ldw, a.K, a.N);
    to_planes(jobs[count++], g.dx, true, a.transpose_w);
  }
  if (dw) {
    // dW = X^T D (or D^T X): columns of both, k over M.
    d.col_shift = g.col_shift;
    to_planes(d, g.dw, !a.transpose_w, true);
    jobs[count] = job_of(a.x, a.ldx, a.M, a.K);
    to_planes(jobs[count++], g.dw, a.transpose_w, true);
  }
  if (count > 0) jobs[count++] = d;

  const bool split_joins = count > 0 && split_jobs_blocks(jobs, count) <= kSplitJoinBlocks;
  err = launch_columns(cols, stream);
  if (err == hipSuccess && !split_joins) err = launch_columns_join(join, stream);
  if (err == hipSuccess && count > 0)
    err = launch_split_jobs(jobs, count, a.scale, stream, split_joins ? &join : nullptr);
  if (err == hipSuccess && outer) {
    const OuterSide x{a.x, a.ldx, a.K, nullptr, 0}, dd{d.s, d.ld, a.N, d.z, d.ldz};
    const OuterArgs o{static_cast<int>(a.M), a.activation, a.transpose_w ? dd : x,
                      a.transpose_w ? x : dd, a.dw, a.lddw};
    err = launch_linear_outer(o, stream);
  }
  if (err == hipSuccess && dx_rows) {
    LinearArgs r{};
    r.M = a.M, r.N = a.K, r.K = a.N;
    r.x = d.s, r.ldx = d.ld;
    r.w = a.w, r.ldw = a.ldw, r.transpose_w = !a.transpose_w;
    r.y = a.dx, r.ldy = a.lddx;
    r.scale = a.scale, r.variant = a.variant;
    err = launch_linear_rows(r, g.row_shift, g.rows, stream);
  } else if (err == hipSuccess && dx) {
    if (dw) {
      const int64_t M[2] = {a.M, dw_rows}, N[2] = {a.K, dw_cols}, K[2] = {a.N, a.M};
      if (const int tile = pair_gemm_tile(M, N, K, a.variant, !scaled_kernel_ok(a.scale))) {
        const Planes p[2] = {g.dx, g.dw};
        float* const C[2] = {a.dx, a.dw};
        const int64_t ldc[2] = {a.lddx, a.lddw};
        const Unscale epi[2] = {ex, ew};
        return launch_gemm_pair(tile, p, M, N, C, ldc, a.scale, a.variant, epi, stream);
      }
    }
    err = launch_gemm_epilogue(g.dx, a.M, a.K, a.dx, a.lddx, a.scale, a.variant, ex, false,
                               stream);
  }
  // As B, D is scaled so that s B_hi is finite where D is, and its words never ask
  // for the fallback (split_tile).
  if (err == hipSuccess && dw)
    err = launch_gemm_epilogue(g.dw, dw_rows, dw_cols, a.dw, a.lddw, a.scale, a.variant, ew,
                               !a.transpose_w, stream);
  return err;
}

}  // namespace sgc
