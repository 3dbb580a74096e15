// AdamW over many tensors in one launch, states in 32 or 8 bits (gfx950).
//
// The formulas are in include/sgemm_cube_layers.h.  Each operation is rounded
// once and none are fused (contraction is off below), so that an 8-bit code
// does not depend on how a compiler pairs them.  8-bit states are coded in
// blocks of 256 values, a wave to a block: four values a lane, the block's
// largest by a reduction over the wave.
#include <algorithm>

#include "layers.h"

#pragma clang fp contract(off)

namespace sgc {
namespace {

constexpr int kThreads = 256;
constexpr int kWaveValues = kAdamwBlock;  // values a wave takes at a time, four a lane
static_assert(kWaveValues == 64 * 4, "a block is a wave's four values a lane");

// One tensor of a launch.  `first`: the first chunk of the grid that is its.
struct Entry {
  float* p;
  const void* g;
  void* m;
  void* v;
  float* ms;
  float* vs;
  int64_t count;
  float keep;  // 1 - lr weight_decay
  uint32_t first;
};

// Tensors of a launch: as many as its arguments hold (4 KiB).
constexpr int kEntries = 48;
constexpr int kWaveBlocks = 4;  // blocks of 256 values that a wave takes in turn
constexpr int kChunk = kThreads / 64 * kWaveBlocks * kWaveValues;  // values a workgroup takes
// Chunks of a launch (a grid holds less than 2^32 threads); the largest tensor fits.
constexpr int64_t kMaxChunks = int64_t{1} << 23;
static_assert(kAdamwMaxCount <= kMaxChunks * kChunk, "a tensor fits a launch");

struct Args {
  AdamwHyper h;
  int entries;
  Entry e[kEntries];
};
static_assert(sizeof(Args) <= 4096, "kernel arguments");

// The entry of chunk `c`: the last whose first chunk is not past it.
__device__ __forceinline__ int entry_of(const Args& a, uint32_t c) {
  int lo = 0, hi = a.entries - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.e[mid].first <= c) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ float grad_of(const void* g, int64_t i, int dtype) {
  if (dtype == kF32) return static_cast<const float*>(g)[i];
  if (dtype == kF16) return static_cast<float>(static_cast<const _Float16*>(g)[i]);
  return static_cast<float>(static_cast<const __bf16*>(g)[i]);
}

// Largest of the wave's values, as bits (non-negative floats, infinities and
// NaN order like their bits); NaN where that is not finite, so that a block which
// has met an infinity stands for NaN throughout, whatever its codes.
__device__ __forceinline__ float wave_max(float v) {
  uint32_t b = __builtin_bit_cast(uint32_t, v);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1)
    b = max(b, static_cast<uint32_t>(__shfl_xor(static_cast<int>(b), off)));
  return __builtin_bit_cast(float, b < 0x7f800000u ? b : 0x7fc00000u);
}

// Largest magnitude of a lane's four values, compared as bits too: a NaN is the
// largest.
__device__ __forceinline__ float largest4(const float (&x)[4]) {
  uint32_t b = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    b = max(b, __builtin_bit_cast(uint32_t, __builtin_fabsf(x[k])));
  return __builtin_bit_cast(float, b);
}

__device__ __forceinline__ float decode_m(int8_t c, float s) {
  const float x = static_cast<float>(c) * (1.0f / 127.0f);
  return (x * __builtin_fabsf(x)) * s;
}
__device__ __forceinline__ float decode_v(uint8_t c, float s) {
  float x = static_cast<float>(c) * (1.0f / 255.0f);
  x = x * x;
  return (x * x) * s;
}
// x / s for a block whose largest is s (0 for a block of zeros).
__device__ __forceinline__ float ratio(float x, float s) { return s > 0.0f ? x / s : 0.0f; }

__device__ __forceinline__ int8_t encode_m(float m, float s) {
  const float c = __builtin_rintf(__builtin_sqrtf(ratio(__builtin_fabsf(m), s)) * 127.0f);
  return static_cast<int8_t>(m < 0.0f ? -c : c);
}
__device__ __forceinline__ uint8_t encode_v(float v, float s) {
  const float c = __builtin_rintf(__builtin_sqrtf(__builtin_sqrtf(ratio(v, s))) * 255.0f);
  return static_cast<uint8_t>(v > 0.0f && c < 1.0f ? 1.0f : c);
}

template <int kBits>
__device__ __forceinline__ void adamw_block(const Entry& e, const AdamwHyper& h, int grad_dtype,
                                            int64_t block) {
  const int64_t i0 = block * kWaveValues + (threadIdx.x & 63) * 4;
  float m[4], v[4];
  float ms = 0.0f, vs = 0.0f;
  if constexpr (kBits == 8) ms = e.ms[block], vs = e.vs[block];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int64_t i = i0 + k;
    m[k] = v[k] = 0.0f;
    if (i >= e.count) continue;
    const float g = grad_of(e.g, i, grad_dtype) * h.grad_scale;
    float m0, v0;
    if constexpr (kBits == 8) {
      m0 = decode_m(static_cast<const int8_t*>(e.m)[i], ms);
      v0 = decode_v(static_cast<const uint8_t*>(e.v)[i], vs);
    } else {
      m0 = static_cast<const float*>(e.m)[i];
      v0 = static_cast<const float*>(e.v)[i];
    }
    m[k] = h.beta1 * m0 + h.rest1 * g;
    v[k] = h.beta2 * v0 + h.rest2 * (g * g);
    const float u = m[k] / (__builtin_sqrtf(v[k]) * h.root + h.eps);
    e.p[i] = e.p[i] * e.keep - h.step_size * u;
    if constexpr (kBits == 32) {
      static_cast<float*>(e.m)[i] = m[k];
      static_cast<float*>(e.v)[i] = v[k];
    }
  }
  if constexpr (kBits == 8) {
    ms = wave_max(largest4(m));
    vs = wave_max(largest4(v));
    if ((threadIdx.x & 63) == 0) e.ms[block] = ms, e.vs[block] = vs;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (i0 + k >= e.count) continue;
      static_cast<int8_t*>(e.m)[i0 + k] = encode_m(m[k], ms);
      static_cast<uint8_t*>(e.v)[i0 + k] = encode_v(v[k], vs);
    }
  }
}

// f(block) for each block of this wave's part of a workgroup's chunk.
template <typename F>
__device__ __forceinline__ void each_block(const Entry& e, F f) {
  const int64_t b0 = (static_cast<int64_t>(blockIdx.x - e.first) * (kThreads / 64) +
                      (threadIdx.x >> 6)) * kWaveBlocks;
  for (int64_t b = b0; b < b0 + kWaveBlocks && b * kWaveValues < e.count; ++b) f(b);
}

template <int kBits>
__global__ __launch_bounds__(kThreads) void adamw_kernel(Args a, int grad_dtype) {
  const Entry& e = a.e[entry_of(a, blockIdx.x)];
  each_block(e, [&](int64_t b) { adamw_block<kBits>(e, a.h, grad_dtype, b); });
}

// What 8-bit states stand for, written where an entry's p and g point.
__global__ __launch_bounds__(kThreads) void values_kernel(Args a) {
  const Entry& e = a.e[entry_of(a, blockIdx.x)];
  float* const vo = static_cast<float*>(const_cast<void*>(e.g));
  each_block(e, [&](int64_t b) {
    const float ms = e.ms[b], vs = e.vs[b];
    const int64_t i0 = b * kWaveValues + (threadIdx.x & 63) * 4;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (i0 + k >= e.count) continue;
      e.p[i0 + k] = decode_m(static_cast<const int8_t*>(e.m)[i0 + k], ms);
      vo[i0 + k] = decode_v(static_cast<const uint8_t*>(e.v)[i0 + k], vs);
    }
  });
}

// Packs the tensors into as few launches as their entries and chunks allow.
template <typename Fill, typename Launch>
hipError_t pack(int64_t tensors, const sgemm_cube_adamw_tensor_t* list, Args& a, Fill fill,
                Launch launch) {
  int64_t chunks = 0;
  a.entries = 0;
  auto flush = [&]() -> hipError_t {
    if (a.entries == 0) return hipSuccess;
    launch(dim3(static_cast<unsigned>(chunks)));
    a.entries = 0;
    chunks = 0;
    return hipGetLastError();
  };
  for (int64_t i = 0; i < tensors; ++i) {
    if (list[i].count == 0) continue;
    const int64_t need = (list[i].count + kChunk - 1) / kChunk;
    if (a.entries == kEntries || chunks + need > kMaxChunks)
      if (const hipError_t err = flush(); err != hipSuccess) return err;
    Entry& e = a.e[a.entries++];
    e.m = list[i].exp_avg;
    e.v = list[i].exp_avg_sq;
    e.ms = list[i].exp_avg_scale;
    e.vs = list[i].exp_avg_sq_scale;
    e.count = list[i].count;
    e.first = static_cast<uint32_t>(chunks);
    fill(e, i);
    chunks += need;
  }
  return flush();
}

}  // namespace

hipError_t launch_adamw(int64_t tensors, const sgemm_cube_adamw_tensor_t* list, int grad_dtype,
                        int state_bits, double lr, const AdamwHyper& h, hipStream_t stream) {
  Args a;
  a.h = h;
  return pack(
      tensors, list, a,
      [&](Entry& e, int64_t i) {
        e.p = list[i].param;
        e.g = list[i].grad;
        e.keep = static_cast<float>(1.0 - lr * list[i].weight_decay);
      },
      [&](dim3 grid) {
        if (state_bits == 8)
          hipLaunchKernelGGL(adamw_kernel<8>, grid, dim3(kThreads), 0, stream, a, grad_dtype);
        else
          hipLaunchKernelGGL(adamw_kernel<32>, grid, dim3(kThreads), 0, stream, a, grad_dtype);
      });
}

hipError_t launch_adamw_values(int64_t tensors, const sgemm_cube_adamw_tensor_t* list,
                               float* const* exp_avg, float* const* exp_avg_sq,
                               hipStream_t stream) {
  Args a;
  a.h = AdamwHyper{};
  return pack(
      tensors, list, a,
      [&](Entry& e, int64_t i) {
        e.p = exp_avg[i];
        e.g = exp_avg_sq[i];
        e.keep = 0.0f;
      },
      [&](dim3 grid) {
        hipLaunchKernelGGL(values_kernel, grid, dim3(kThreads), 0, stream, a);
      });
}

}  // namespace sgc
