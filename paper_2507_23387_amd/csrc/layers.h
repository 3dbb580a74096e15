// Internal declarations of the layer kernels (layer norm, AdamW, linear); the
// public interface is include/sgemm_cube_layers.h.
#pragma once

#include "internal.h"
#include "sgemm_cube_layers.h"

namespace sgc {

// Element types of the layers' operands (sgemm_cube_dtype_t).
enum Dtype : int { kF32 = 0, kF16 = 1, kBF16 = 2 };
inline int dtype_bytes(int dtype) { return dtype == kF32 ? 4 : 2; }

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
