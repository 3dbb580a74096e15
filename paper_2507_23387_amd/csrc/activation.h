// The activations of a linear layer's epilogue and their derivatives.  Internal.
#pragma once

#include <hip/hip_runtime.h>

#include "sgemm_cube_layers.h"

namespace sgc {
namespace {

// 1 / (1 + exp(-x)) on the hardware's exp2 and reciprocal, one unit in the last
// place each; the rounded exponent adds |x| 2^-24, which counts only where the
// result is small.
__device__ __forceinline__ float sigmoid(float x) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * x));
}

// 2 sqrt(2 / pi) (z + 0.044715 z^3): gelu_tanh(z) = z sigmoid(that).
__device__ __forceinline__ float gelu_tanh_arg(float z) {
  constexpr float kC = 1.59576912f;
  return z * (kC + (kC * 0.044715f) * z * z);
}

__device__ __forceinline__ float activate(int activation, float z) {
  switch (activation) {
    case SGEMM_CUBE_ACT_RELU: return z < 0.0f ? 0.0f : z;
    case SGEMM_CUBE_ACT_GELU: return 0.5f * z * (1.0f + erff(0.707106781f * z));
    case SGEMM_CUBE_ACT_GELU_TANH: return z * sigmoid(gelu_tanh_arg(z));
    case SGEMM_CUBE_ACT_SILU: return z * sigmoid(z);
    default: return z;
  }
}

__device__ __forceinline__ float activate_grad(int activation, float z) {
  switch (activation) {
    case SGEMM_CUBE_ACT_RELU: return z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z;  // NaN stays
    case SGEMM_CUBE_ACT_GELU: {
      const float density = 0.398942280f * __builtin_amdgcn_exp2f(-0.721347520f * z * z);
      return 0.5f * (1.0f + erff(0.707106781f * z)) + z * density;
    }
    case SGEMM_CUBE_ACT_GELU_TANH: {
      constexpr float kC = 1.59576912f;
      const float s = sigmoid(gelu_tanh_arg(z));
      return s + z * s * (1.0f - s) * (kC + (3.0f * kC * 0.044715f) * z * z);
    }
    case SGEMM_CUBE_ACT_SILU: {
      const float s = sigmoid(z);
      return s + z * s * (1.0f - s);
    }
    default: return 1.0f;
  }
}

}  // namespace
}  // namespace sgc
