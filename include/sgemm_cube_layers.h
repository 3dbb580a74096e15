/*
 * sgemm_cube_layers.h -- the layers around the FP32-accuracy GEMM of
 * sgemm_cube.h, on AMD Instinct MI355X (gfx950).
 *
 * Conventions of sgemm_cube.h hold: row-major matrices with leading
 * dimensions in elements, device pointers owned by the caller, asynchronous
 * calls on `stream` whose argument errors are reported before any device work,
 * its status codes, no allocation and no state kept between calls.  Operands
 * overlap where the memory from their first to their last entry does, so also
 * as columns side by side in one buffer.  Sums and statistics are held in 32
 * bits, in an order that depends on the sizes alone, so a call repeated on the
 * same operands gives the same bits.  (One exception: a replay of a captured
 * linear or linear_backward, after an earlier one whose W or X had entries past
 * 65504 / scale, stays with the kernels that those need, which round differently.)
 */
#ifndef SGEMM_CUBE_LAYERS_H_
#define SGEMM_CUBE_LAYERS_H_

#include "sgemm_cube.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Activations, and their derivatives in the backward pass. */
typedef enum {
  SGEMM_CUBE_ACT_NONE = 0,
  SGEMM_CUBE_ACT_RELU = 1,      /* max(z, 0), derivative 0 at 0 */
  SGEMM_CUBE_ACT_GELU = 2,      /* z Phi(z), Phi the normal distribution to 3 units of
                                   2^-24, and to 1e-5 of itself from -8 on */
  SGEMM_CUBE_ACT_GELU_TANH = 3, /* z (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) / 2 */
  SGEMM_CUBE_ACT_SILU = 4       /* z / (1 + exp(-z)) */
} sgemm_cube_activation_t;

/*
 * A linear layer with its epilogue:
 *   Z = X W + bias,   Y = act(Z) + R,
 * the product by the three-product method of sgemm_cube.h, the epilogue in 32
 * bits.
 *   M, N, K      >= 0.  M == 0 or N == 0: nothing is done.  K == 0: X W = 0.
 *   X, ldx       row-major M x K, ldx >= max(1, K).
 *   W, ldw       transpose_w == 0: row-major K x N, ldw >= max(1, N);
 *                otherwise row-major N x K (its rows the outputs), ldw >=
 *                max(1, K).
 *   bias         NULL, or N values.
 *   activation   sgemm_cube_activation_t.
 *   R, ldr       NULL, or row-major M x N, ldr >= max(1, N) (ignored without R).
 *                May be Y itself (same pointer and leading dimension).
 *   Y, ldy       row-major M x N, ldy >= max(1, N).
 *   Z, ldz       NULL, or row-major M x N that receives Z, what the backward
 *                pass needs of a layer with an activation.
 *   scale, accum_order  as for sgemm_cube.  Results of few rows or columns (up to
 *                128, or 256 where there are few entries) are computed from FP32
 *                operands directly, the sums termwise whatever the order.
 *   ws, ws_bytes at least sgemm_cube_linear_workspace_size(M, N, K) bytes,
 *                256-byte aligned, as for sgemm_cube_ws.
 * Outputs must not overlap each other, an input or the workspace, but for R.
 * As for sgemm_cube there is no range guard: entries of X and W with a
 * magnitude of 65520 or more give infinities or NaN in their rows and columns,
 * and entries below 2^-14 are off by up to 2^-36 and not by 2^-22 of themselves.
 * There is no pre-scaling or range report here (sgemm_cube_ex has both).
 */
int sgemm_cube_linear(int64_t M, int64_t N, int64_t K, const float* X, int64_t ldx,
                      const float* W, int64_t ldw, int transpose_w, const float* bias,
                      int activation, const float* R, int64_t ldr, float* Y, int64_t ldy,
                      float* Z, int64_t ldz, float scale, int accum_order, void* ws,
                      size_t ws_bytes, hipStream_t stream);
size_t sgemm_cube_linear_workspace_size(int64_t M, int64_t N, int64_t K);

/*
 * Gradients of the linear layer: with D = dY act'(Z), entry by entry,
 *   dX = D W^T,   dW = X^T D,   dbias_j = sum_i D_ij
 * (the residual's gradient is dY itself).  Gradients are often far below what
 * FP16 holds, so before it is split D is multiplied by powers of two, for dX one
 * for each row and for dW one for each column, found from the line's largest finite
 * magnitude, and dX and dW are scaled back: a line far below the others keeps its
 * digits, and within one an entry is off by at most 2^-38 of the line's largest (or
 * 2^-22 of itself).  X and W are taken as they are, as in the forward pass.  (dW of
 * few rows is summed in FP32 without a split.)
 *   dY, lddy     row-major M x N.
 *   Z, ldz       row-major M x N; NULL (and ldz ignored) without an activation.
 *   X, W         as in the forward pass.
 *   dX, lddx     NULL, or row-major M x K, overwritten.
 *   dW, lddw     NULL, or of W's shape and layout, overwritten (zeros for M == 0).
 *   dbias        NULL, or N values, overwritten (zeros for M == 0).
 *   ws, ws_bytes at least sgemm_cube_linear_backward_workspace_size(M, N, K)
 *                bytes, 256-byte aligned, as for sgemm_cube_ws.
 * Outputs must not overlap each other, an input or the workspace.
 */
int sgemm_cube_linear_backward(int64_t M, int64_t N, int64_t K, const float* dY, int64_t lddy,
                               const float* Z, int64_t ldz, const float* X, int64_t ldx,
                               const float* W, int64_t ldw, int transpose_w, int activation,
                               float* dX, int64_t lddx, float* dW, int64_t lddw, float* dbias,
                               float scale, int accum_order, void* ws, size_t ws_bytes,
                               hipStream_t stream);
size_t sgemm_cube_linear_backward_workspace_size(int64_t M, int64_t N, int64_t K);

/* Element types of a layer norm's rows. */
typedef enum {
  SGEMM_CUBE_F32 = 0,
  SGEMM_CUBE_F16 = 1,
  SGEMM_CUBE_BF16 = 2
} sgemm_cube_dtype_t;

/*
 * Layer norm of each row: with mu the row's mean and
 * r = 1 / sqrt(mean((x - mu)^2) + eps),
 *   Y_ij = (X_ij - mu_i) r_i weight_j + bias_j,
 * computed in 32 bits and rounded once to the element type.
 *
 *   rows, cols   >= 0; nothing is done where either is 0, except that rows
 *                without columns get NaN in mean and rstd.
 *   dtype        sgemm_cube_dtype_t of X and Y.
 *   X, ldx       row-major rows x cols, ldx >= max(1, cols).
 *   weight, bias FP32, cols values each; NULL: all ones, all zeros.
 *   eps          finite, >= 0.  (With eps = 0 a row of equal values has no result:
 *                it gives NaN, or its mean's rounding error over itself.)
 *   Y, ldy       row-major rows x cols; may be X itself (same pointer and
 *                leading dimension), otherwise must not overlap X.
 *   mean, rstd   NULL, or rows FP32 values each that receive mu and r.
 * A NaN or an infinity in a row gives NaN in that row alone.
 */
int sgemm_cube_layer_norm(int64_t rows, int64_t cols, int dtype, const void* X, int64_t ldx,
                          const float* weight, const float* bias, float eps, void* Y,
                          int64_t ldy, float* mean, float* rstd, hipStream_t stream);

/*
 * Gradients of the layer norm: with h_ij = (X_ij - mean_i) rstd_i and
 * g_ij = dY_ij weight_j,
 *   dX_ij      = rstd_i (g_ij - mean_j(g_ij) - h_ij mean_j(g_ij h_ij))
 *   dweight_j  = sum_i dY_ij h_ij
 *   dbias_j    = sum_i dY_ij.
 *   dY, X, dX    of type dtype, row-major with leading dimensions lddy, ldx,
 *                lddx >= max(1, cols).  dX may be dY itself (same pointer and
 *                leading dimension), otherwise must not overlap an input.
 *   weight       NULL: all ones.
 *   mean, rstd   what the forward call gave for the same X.
 *   dweight, dbias   FP32, cols values each, overwritten (zeros for rows == 0);
 *                either or both may be NULL.
 *   ws, ws_bytes at least sgemm_cube_layer_norm_backward_workspace_size(rows,
 *                cols) bytes, 256-byte aligned, as for sgemm_cube_ws.
 */
int sgemm_cube_layer_norm_backward(int64_t rows, int64_t cols, int dtype, const void* dY,
                                   int64_t lddy, const void* X, int64_t ldx, const float* weight,
                                   const float* mean, const float* rstd, void* dX, int64_t lddx,
                                   float* dweight, float* dbias, void* ws, size_t ws_bytes,
                                   hipStream_t stream);
size_t sgemm_cube_layer_norm_backward_workspace_size(int64_t rows, int64_t cols);

/* Values of an 8-bit AdamW state that share a scale. */
enum { SGEMM_CUBE_ADAMW_BLOCK = 256 };

/*
 * One tensor of an AdamW step: `count` adjacent values.  States of 32 bits are
 * FP32 and the scales NULL.  States of 8 bits are int8 codes c for exp_avg and
 * uint8 codes for exp_avg_sq with an FP32 scale s per block of
 * SGEMM_CUBE_ADAMW_BLOCK values (the last block may be shorter), and stand for
 *   exp_avg:    s (c / 127) |c / 127|, s the block's largest magnitude
 *   exp_avg_sq: s (c / 255)^4,         s the block's largest value
 * so that both keep their small values: codes all zero with any scale, or any
 * codes with scale 0, are a state of zeros.
 */
typedef struct {
  int64_t count;
  float* param;
  const void* grad; /* of type grad_dtype */
  void* exp_avg;
  void* exp_avg_sq;
  float* exp_avg_scale;
  float* exp_avg_sq_scale;
  double weight_decay;
} sgemm_cube_adamw_tensor_t;

/*
 * An AdamW step over all tensors of the list, in place: with g' = grad_scale g,
 *   m = beta1 m + (1 - beta1) g'
 *   v = beta2 v + (1 - beta2) g' g'
 *   p = p (1 - lr weight_decay)
 *       - lr / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps)
 * in 32 bits, each operation rounded once.  8-bit states are decoded, stepped
 * and encoded again: c = round(127 sqrt(|m| / s)) with m's sign, and
 * round(255 sqrt(sqrt(v / s))), at least 1 where v > 0, so that no value that
 * has been seen divides by eps alone; the step itself uses m and v before they
 * are encoded.  A NaN or an infinity among a block's gradients makes its state
 * NaN.
 *   tensors, list   a HOST array, read during the call; entries of count 0 are
 *                   skipped.  Operands of one entry must not overlap, nor those
 *                   of different entries (only the former is checked).
 *   grad_dtype      sgemm_cube_dtype_t of every gradient.
 *   state_bits      8 or 32.
 *   step            >= 1, the number of this step.  A captured call keeps it, and so
 *                   both powers of beta, on every replay.
 */
int sgemm_cube_adamw(int64_t tensors, const sgemm_cube_adamw_tensor_t* list, int grad_dtype,
                     int state_bits, double lr, double beta1, double beta2, double eps,
                     double grad_scale, int64_t step, hipStream_t stream);

/*
 * What 8-bit states stand for, as a checkpoint holds them: exp_avg[i] and
 * exp_avg_sq[i] (HOST arrays of device pointers, read during the call) receive
 * list[i].count FP32 values each.  param and grad are not read.
 */
int sgemm_cube_adamw_values(int64_t tensors, const sgemm_cube_adamw_tensor_t* list,
                            float* const* exp_avg, float* const* exp_avg_sq, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* SGEMM_CUBE_LAYERS_H_ */
