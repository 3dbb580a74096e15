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

// The normal distribution Phi(z), and e = exp(-z^2 / 2): with x = |z| and
// w = p x / (1 + p x), Phi(-x) = e M(w), M = exp(x^2 / 2) Phi(-x) a smooth function of w
// that falls from 1/2 at 0 to 0 at 1.  M - 1/2 is w times a polynomial of degree 7,
// fitted over x <= 16 by linear programming so that the largest of |error| e and of
// |error| / (30 M) is least: 0.085 units of 2^-24.  Each step's rounding is that of a
// value that e or w makes small, so that Phi is off by less than 3 units in all (1.3
// where the reciprocal and exp2 are rounded once), and by 1e-5 of itself down to z = -8.
// 19 instructions.  The library's erff, both of its branches taken by a wave, is some
// 80, which cost the epilogue of a 256 x 256 tile more than its stores.  (x stays
// finite, so that w does; e is 0 long before 20.)
__device__ __forceinline__ float normal_cdf(float z, float& e) {
  const float x = 0.2275f * __builtin_fminf(__builtin_fabsf(z), 20.0f);
  const float w = x * __builtin_amdgcn_rcpf(1.0f + x);
  float p = __builtin_fmaf(-0.0837816373f, w, 0.345369846f);
  p = __builtin_fmaf(p, w, -0.407096118f);
  p = __builtin_fmaf(p, w, -0.471546352f);
  p = __builtin_fmaf(p, w, 2.17985702f);
  p = __builtin_fmaf(p, w, -3.38594103f);
  p = __builtin_fmaf(p, w, 3.0766933f);
  p = __builtin_fmaf(p, w, -1.75359154f);
  e = __builtin_amdgcn_exp2f(-0.721347520f * z * z);
  const float q = __builtin_fmaf(p, w, 0.5f) * e;
  return z < 0.0f ? q : 1.0f - q;
}

__device__ __forceinline__ float activate(int activation, float z) {
  float e;
  switch (activation) {
    case SGEMM_CUBE_ACT_RELU: return z < 0.0f ? 0.0f : z;
    case SGEMM_CUBE_ACT_GELU: return z * normal_cdf(z, e);
    case SGEMM_CUBE_ACT_GELU_TANH: return z * sigmoid(gelu_tanh_arg(z));
    case SGEMM_CUBE_ACT_SILU: return z * sigmoid(z);
    default: return z;
  }
}

// The same for kU pieces of four values behind one branch.
template <typename V, int kU>
__device__ __forceinline__ void activate_all(int activation, V (&v)[kU]) {
  auto each = [&](auto f) {
#pragma unroll
    for (int u = 0; u < kU; ++u)
#pragma unroll
      for (int k = 0; k < 4; ++k) v[u][k] = f(v[u][k]);
  };
  switch (activation) {
    case SGEMM_CUBE_ACT_RELU:
      each([](float z) { return activate(SGEMM_CUBE_ACT_RELU, z); });
      break;
    case SGEMM_CUBE_ACT_GELU:
      each([](float z) { return activate(SGEMM_CUBE_ACT_GELU, z); });
      break;
    case SGEMM_CUBE_ACT_GELU_TANH:
      each([](float z) { return activate(SGEMM_CUBE_ACT_GELU_TANH, z); });
      break;
    case SGEMM_CUBE_ACT_SILU:
      each([](float z) { return activate(SGEMM_CUBE_ACT_SILU, z); });
      break;
    default: break;
  }
}

__device__ __forceinline__ float activate_grad(int activation, float z) {
  switch (activation) {
    case SGEMM_CUBE_ACT_RELU: return z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z;  // NaN stays
    case SGEMM_CUBE_ACT_GELU: {
      float e;
      const float phi = normal_cdf(z, e);
      return phi + z * 0.398942280f * e;
    }
    case SGEMM_CUBE_ACT_GELU_TANH: {
      constexpr float kC = 1.59576912f;
      const float s = sigmoid(gelu_tanh_arg(z));
      // z^2 stays finite where s (1 - s) is 0.
      const float zz = __builtin_fminf(z * z, 1e30f);
      return s + z * s * (1.0f - s) * (kC + (3.0f * kC * 0.044715f) * zz);
    }
    case SGEMM_CUBE_ACT_SILU: {
      const float s = sigmoid(z);
      return s + z * s * (1.0f - s);
    }
    default: return 1.0f;
  }
}

// d *= act'(z) for kU pieces behind one branch.
template <typename V, int kU>
__device__ __forceinline__ void multiply_grad(int activation, V (&d)[kU], const V (&z)[kU]) {
  auto each = [&](auto f) {
#pragma unroll
    for (int u = 0; u < kU; ++u)
#pragma unroll
      for (int k = 0; k < 4; ++k) d[u][k] *= f(z[u][k]);
  };
  switch (activation) {
    case SGEMM_CUBE_ACT_RELU:
      each([](float x) { return activate_grad(SGEMM_CUBE_ACT_RELU, x); });
      break;
    case SGEMM_CUBE_ACT_GELU:
      each([](float x) { return activate_grad(SGEMM_CUBE_ACT_GELU, x); });
      break;
    case SGEMM_CUBE_ACT_GELU_TANH:
      each([](float x) { return activate_grad(SGEMM_CUBE_ACT_GELU_TANH, x); });
      break;
    case SGEMM_CUBE_ACT_SILU:
      each([](float x) { return activate_grad(SGEMM_CUBE_ACT_SILU, x); });
      break;
    default: break;
  }
}

}  // namespace
}  // namespace sgc
