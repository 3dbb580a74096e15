// Layer norm of rows and its gradients (gfx950).
//
// Forward, per row: mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps),
// y = (x - mu) r w + b.  The variance is formed from the centred values, so a
// row whose mean is large against its spread keeps its digits.
// Backward, with h = (x - mu) r and g = dy w, per row:
// dx = r (g - mean(g) - h mean(g h)); over the rows: dw = sum dy h, db = sum dy.
// All sums are FP32 and have an order that the sizes alone fix.
#include <algorithm>

#include "layers.h"

namespace sgc {
namespace {

template <int kDtype>
struct Elem;
template <>
struct Elem<kF32> {
  typedef float T;
};
template <>
struct Elem<kF16> {
  typedef _Float16 T;
};
template <>
struct Elem<kBF16> {
  typedef __bf16 T;
};

constexpr int kThreads = 256;

// Sum over the workgroup's threads, the same bits in each.
__device__ __forceinline__ float block_sum(float v, float* lds) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// A workgroup per row, three passes over it.
template <int kDtype>
__global__ __launch_bounds__(kThreads) void norm_kernel(NormArgs a) {
  typedef typename Elem<kDtype>::T T;
  __shared__ float lds[kThreads / 64];
  for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + i * a.ldx;
    T* y = static_cast<T*>(a.y) + i * a.ldy;
    float s = 0.0f;
    for (int64_t j = threadIdx.x; j < a.cols; j += kThreads) s += static_cast<float>(x[j]);
    const float mu = block_sum(s, lds) / static_cast<float>(a.cols);
    s = 0.0f;
    for (int64_t j = threadIdx.x; j < a.cols; j += kThreads) {
      const float d = static_cast<float>(x[j]) - mu;
      s += d * d;
    }
    const float r = 1.0f / __builtin_sqrtf(block_sum(s, lds) / static_cast<float>(a.cols) + a.eps);
    for (int64_t j = threadIdx.x; j < a.cols; j += kThreads) {
      const float h = (static_cast<float>(x[j]) - mu) * r;
      y[j] = static_cast<T>(h * (a.weight ? a.weight[j] : 1.0f) + (a.bias ? a.bias[j] : 0.0f));
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[i] = mu;
      if (a.rstd) a.rstd[i] = r;
    }
  }
}

// dX, a workgroup per row.
template <int kDtype>
__global__ __launch_bounds__(kThreads) void norm_dx_kernel(NormGradArgs a) {
  typedef typename Elem<kDtype>::T T;
  __shared__ float lds[kThreads / 64];
  for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + i * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + i * a.lddy;
    T* dx = static_cast<T*>(a.dx) + i * a.lddx;
    const float mu = a.mean[i], r = a.rstd[i];
    float s1 = 0.0f, s2 = 0.0f;
    for (int64_t j = threadIdx.x; j < a.cols; j += kThreads) {
      const float g = static_cast<float>(dy[j]) * (a.weight ? a.weight[j] : 1.0f);
      s1 += g;
      s2 += g * ((static_cast<float>(x[j]) - mu) * r);
    }
    s1 = block_sum(s1, lds) / static_cast<float>(a.cols);
    s2 = block_sum(s2, lds) / static_cast<float>(a.cols);
    for (int64_t j = threadIdx.x; j < a.cols; j += kThreads) {
      const float g = static_cast<float>(dy[j]) * (a.weight ? a.weight[j] : 1.0f);
      const float h = (static_cast<float>(x[j]) - mu) * r;
      dx[j] = static_cast<T>(r * (g - s1 - h * s2));
    }
  }
}

// Column sums of one slab of rows (blockIdx.y), a thread per column.
template <int kDtype>
__global__ __launch_bounds__(kThreads) void norm_dw_kernel(NormGradArgs a, int64_t slab_rows) {
  typedef typename Elem<kDtype>::T T;
  const int64_t j = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (j >= a.cols) return;
  const int64_t i0 = blockIdx.y * slab_rows, i1 = min(a.rows, i0 + slab_rows);
  float dw = 0.0f, db = 0.0f;
  for (int64_t i = i0; i < i1; ++i) {
    const float dy = static_cast<float>(static_cast<const T*>(a.dy)[i * a.lddy + j]);
    const float x = static_cast<float>(static_cast<const T*>(a.x)[i * a.ldx + j]);
    dw += dy * ((x - a.mean[i]) * a.rstd[i]);
    db += dy;
  }
  a.partial[(2 * blockIdx.y) * a.cols + j] = dw;
  a.partial[(2 * blockIdx.y + 1) * a.cols + j] = db;
}

__global__ __launch_bounds__(kThreads) void norm_join_kernel(const float* __restrict__ partial,
                                                             int64_t slabs, int64_t cols,
                                                             float* dweight, float* dbias) {
  const int64_t j = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (j >= cols) return;
  float dw = 0.0f, db = 0.0f;
  for (int64_t s = 0; s < slabs; ++s) {
    dw += partial[2 * s * cols + j];
    db += partial[(2 * s + 1) * cols + j];
  }
  if (dweight) dweight[j] = dw;
  if (dbias) dbias[j] = db;
}

unsigned row_grid(int64_t rows) {
  return static_cast<unsigned>(std::min<int64_t>(rows, int64_t{1} << 20));
}

template <int kDtype>
hipError_t grad(const NormGradArgs& a, hipStream_t stream) {
  // The column sums first: dX may be dY.
  if (a.dweight || a.dbias) {
    const int64_t slabs = norm_slabs(a.rows, a.cols);
    const unsigned strips = static_cast<unsigned>((a.cols + kThreads - 1) / kThreads);
    if (slabs > 0) {
      const int64_t slab_rows = (a.rows + slabs - 1) / slabs;
      hipLaunchKernelGGL(norm_dw_kernel<kDtype>, dim3(strips, static_cast<unsigned>(slabs)),
                         dim3(kThreads), 0, stream, a, slab_rows);
      if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(norm_join_kernel, dim3(strips), dim3(kThreads), 0, stream, a.partial,
                       slabs, a.cols, a.dweight, a.dbias);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (a.rows == 0) return hipSuccess;
  hipLaunchKernelGGL(norm_dx_kernel<kDtype>, dim3(row_grid(a.rows)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

int64_t norm_slabs(int64_t rows, int64_t cols) {
  (void)cols;
  return std::min<int64_t>(rows, 256);
}

hipError_t launch_norm(const NormArgs& a, int dtype, hipStream_t stream) {
  const dim3 grid(row_grid(a.rows));
  switch (dtype) {
    case kF32: hipLaunchKernelGGL(norm_kernel<kF32>, grid, dim3(kThreads), 0, stream, a); break;
    case kF16: hipLaunchKernelGGL(norm_kernel<kF16>, grid, dim3(kThreads), 0, stream, a); break;
    case kBF16: hipLaunchKernelGGL(norm_kernel<kBF16>, grid, dim3(kThreads), 0, stream, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_norm_grad(const NormGradArgs& a, int dtype, hipStream_t stream) {
  switch (dtype) {
    case kF32: return grad<kF32>(a, stream);
    case kF16: return grad<kF16>(a, stream);
    case kBF16: return grad<kBF16>(a, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace sgc
