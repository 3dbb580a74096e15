// Internal declarations of the layer kernels (layer norm, AdamW, linear); the
// public interface is include/sgemm_cube_layers.h.
#pragma once

#include "internal.h"
#include "sgemm_cube_layers.h"

namespace sgc {

// Element types of the layers' operands (sgemm_cube_dtype_t).
enum Dtype : int { kF32 = 0, kF16 = 1, kBF16 = 2 };
inline int dtype_bytes(int dtype) { return dtype == kF32 ? 4 : 2; }

// --- linear layer ---------------------------------------------------------------

// One matrix of a split launch: S is rows x cols row-major, times act'(Z) where z
// is not null.  Its planes with S's rows as rows (k = cols) go to row_*, those
// with its columns as rows (k = rows) to col_*; either may be null.  kp_row =
// cols and kp_col = rows rounded up to 64.  Where the planes have shifts, one for
// each of S's rows (columns; read up to a multiple of 64, of 128, whatever is there),
// the values are first multiplied by 2^shift.
// `range`: the header of B-side planes, whose flag words get `stamp` as
// launch_split's do (null: none), but with shifts never say that s B_hi overflows.
struct SplitJob {
  const float* s;
  int64_t ld;
  const float* z;
  int64_t ldz;
  int activation;
  int64_t rows, cols;
  uint16_t* row_hi;
  uint16_t* row_lo;
  uint16_t* col_hi;
  uint16_t* col_lo;
  const int* row_shift;
  const int* col_shift;
  uint32_t* row_range;
  uint32_t* col_range;
  uint32_t row_stamp, col_stamp;
};
constexpr int kSplitJobs = 3;
// The join of what launch_columns left: for each of D's M rows and N columns the
// shift that brings its largest finite magnitude to 2^target (prescale_shift), and
// the sums of the columns.  Null: not wanted.  A split launch can do it on the way:
// each workgroup of the job with shifts finds those of its tile, the first of a line
// also writing them, and workgroups of their own add up dbias.
struct ColumnJoin {
  int64_t M, N;
  int pieces, slabs;
  const float* row_top;  // pieces x M
  const float* col_top;  // slabs x N rounded up to kColumnStrip
  const float* sums;     // slabs x N
  int row_target, col_target;
  int* row_shift;
  int* col_shift;
  float* dbias;
};
hipError_t launch_split_jobs(const SplitJob* jobs, int count, float scale, hipStream_t stream,
                             const ColumnJoin* join = nullptr);
// Workgroups of such a launch without the join's own.
int64_t split_jobs_blocks(const SplitJob* jobs, int count);

// One pass over D = dY act'(Z): for each slab of rows the sums and the largest finite
// magnitudes of D's columns, and for each half of a strip of columns the largest finite
// magnitudes of its rows (ColumnJoin's arrays; null: not wanted).
constexpr int kColumnStrip = 128;
int64_t column_slabs(int64_t M, int64_t N);
int64_t column_strips(int64_t N);
inline int64_t row_pieces(int64_t N) { return 2 * column_strips(N); }
struct ColumnArgs {
  int64_t M, N;
  const float* dy;
  int64_t lddy;
  const float* z;  // null: D = dY
  int64_t ldz;
  int activation;
  float* row_top;
  float* col_top;
  float* sums;
  float* d;  // null, or M x N that receives D
};
hipError_t launch_columns(const ColumnArgs& a, hipStream_t stream);
hipError_t launch_columns_join(const ColumnJoin& j, hipStream_t stream);

// What follows a product P: Y = act(Z) + R, Z = P + bias.
struct Epilogue {
  const float* bias;  // null: none
  int activation;
  const float* r;     // null: none
  int64_t ldr;
  float* z;           // null: not kept
  int64_t ldz;
};
// A gradient's product: row i (or column i) of P times 2^-shift[i].
struct Unscale {
  const int* shift;
  bool columns;
};
// The epilogue where K = 0: P = 0.
hipError_t launch_epilogue(const Epilogue& e, int64_t M, int64_t N, float* Y, int64_t ldy,
                           hipStream_t stream);

// launch_gemm, launch_gemm_small and launch_gemm_unscaled with an epilogue (Epi:
// Epilogue or Unscale); the product's bits are theirs.  C may be the residual.
// no_overflow: the range words say that s B_hi is finite, whatever its values, so
// that the scaled kernels need no fallback.
template <class Epi>
hipError_t launch_gemm_epilogue(const Planes& p, int64_t M, int64_t N, float* C, int64_t ldc,
                                float scale, int variant, const Epi& epi, bool no_overflow,
                                hipStream_t stream);
template <class Epi>
hipError_t launch_gemm_small_epilogue(int tile, const Planes& p, int64_t M, int64_t N, float* C,
                                      int64_t ldc, float scale, int variant, const Epi& epi,
                                      hipStream_t stream);
template <class Epi>
hipError_t launch_gemm_unscaled_epilogue(const Planes& p, int64_t M, int64_t N, float* C,
                                         int64_t ldc, float scale, int variant, bool only,
                                         const Epi& epi, hipStream_t stream);

// launch_gemm_fused_a with an epilogue (requires splits_a_in_gemm).
hipError_t launch_gemm_fused_a_epilogue(const Planes& p, int64_t M, int64_t N, int64_t K,
                                        const float* A, int64_t lda, float* C, int64_t ldc,
                                        float scale, int variant, const Epilogue& epi,
                                        hipStream_t stream);

// Two gradients' products in one launch, on tiles of 32, 64 or 128.
// pair_gemm_tile: the tile where that takes less time than two launches, or 0.
int pair_gemm_tile(const int64_t (&M)[2], const int64_t (&N)[2], const int64_t (&K)[2],
                   int variant, bool unscaled);
hipError_t launch_gemm_pair(int tile, const Planes (&p)[2], const int64_t (&M)[2],
                            const int64_t (&N)[2], float* const (&C)[2], const int64_t (&ldc)[2],
                            float scale, int variant, const Unscale (&epi)[2],
                            hipStream_t stream);

struct LinearArgs {
  int64_t M, N, K;
  const float* x;
  int64_t ldx;
  const float* w;
  int64_t ldw;
  bool transpose_w;
  Epilogue e;
  float* y;
  int64_t ldy;
  float scale;
  int variant;
};

// The linear layer for few rows or few columns (linear_rows.hip), its sums termwise
// whatever the variant.  linear_by_rows, linear_by_columns: the rules that choose
// them.  With `row_shift`, row i of x, a gradient, is multiplied by 2^row_shift[i] as
// it is split, and the result is freed of it again.  The workspace of N columns is
// that of as many rows, linear_rows_ws(N, M, K).
bool linear_by_rows(int64_t M, int64_t N);
bool linear_by_columns(int64_t M, int64_t N);
size_t linear_rows_ws(int64_t M, int64_t N, int64_t K);
hipError_t launch_linear_rows(const LinearArgs& a, const int* row_shift, void* ws,
                              hipStream_t stream);
hipError_t launch_linear_columns(const LinearArgs& a, void* ws, hipStream_t stream);

// out = L^T R in FP32, L and R of M <= kOuterRows rows; a side with z is p times
// act'(z).
constexpr int kOuterRows = 24;
struct OuterSide {
  const float* p;
  int64_t ld, cols;
  const float* z;  // null: p
  int64_t ldz;
};
struct OuterArgs {
  int M, activation;
  OuterSide left, right;
  float* out;  // left.cols x right.cols
  int64_t ldo;
};
hipError_t launch_linear_outer(const OuterArgs& g, hipStream_t stream);

size_t linear_ws(int64_t M, int64_t N, int64_t K);
hipError_t launch_linear(const LinearArgs& a, void* ws, hipStream_t stream);

struct LinearGradArgs {
  int64_t M, N, K;
  const float* dy;
  int64_t lddy;
  const float* z;  // null: no activation
  int64_t ldz;
  const float* x;
  int64_t ldx;
  const float* w;
  int64_t ldw;
  bool transpose_w;
  int activation;
  float* dx;  // null: not wanted, as dw and dbias
  int64_t lddx;
  float* dw;
  int64_t lddw;
  float* dbias;
  float scale;
  int variant;
};
size_t linear_grad_ws(int64_t M, int64_t N, int64_t K);
hipError_t launch_linear_grad(const LinearGradArgs& a, void* ws, hipStream_t stream);

struct NormArgs {
  int64_t rows, cols;
  const void* x;
  int64_t ldx;
  const float* weight;  // null: ones
  const float* bias;    // null: zeros (forward)
  float eps;
  void* y;
  int64_t ldy;
  float* mean;  // forward: may be null
  float* rstd;
};

struct NormGradArgs {
  int64_t rows, cols;
  const void* dy;
  int64_t lddy;
  const void* x;
  int64_t ldx;
  const float* weight;  // null: ones
  const float* mean;
  const float* rstd;
  void* dx;
  int64_t lddx;
  float* dweight;  // may be null
  float* dbias;    // may be null
  float* partial;  // workspace: norm_slabs(rows, cols) x 2 x cols
};

// Slabs of rows whose column sums are formed apart and joined afterwards.
int64_t norm_slabs(int64_t rows, int64_t cols);

hipError_t launch_norm(const NormArgs& a, int dtype, hipStream_t stream);
hipError_t launch_norm_grad(const NormGradArgs& a, int dtype, hipStream_t stream);

// Values of an 8-bit state that share a scale.
constexpr int kAdamwBlock = SGEMM_CUBE_ADAMW_BLOCK;
// More than 288 GB hold: 4 bytes of parameter, 2 of gradient and 2 of state.
constexpr int64_t kAdamwMaxCount = int64_t{1} << 35;

// An AdamW step's numbers in the 32 bits that the kernel works in, each rounded
// once from 64: rest = 1 - beta, step_size = lr / (1 - beta1^t), root =
// 1 / sqrt(1 - beta2^t).
struct AdamwHyper {
  float beta1, rest1, beta2, rest2, eps, grad_scale, step_size, root;
};

hipError_t launch_adamw(int64_t tensors, const sgemm_cube_adamw_tensor_t* list, int grad_dtype,
                        int state_bits, double lr, const AdamwHyper& h, hipStream_t stream);
hipError_t launch_adamw_values(int64_t tensors, const sgemm_cube_adamw_tensor_t* list,
                               float* const* exp_avg, float* const* exp_avg_sq,
                               hipStream_t stream);

}  // namespace sgc
