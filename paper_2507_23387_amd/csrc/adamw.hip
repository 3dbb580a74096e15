// AdamW over many tensors in one launch, states in 32 or 8 bits (gfx950).
//
// The formulas are in include/sgemm_cube_layers.h.  Each operation is rounded
// once and none are fused (contraction is off below), so that an 8-bit code
// does not depend on how a compiler pairs them.  8-bit states are coded in
// blocks of 256 values, a wave to a block: four values a lane, the block's
// largest by a reduction over the wave.
#include <algorithm>
#include <type_traits>

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

// A lane's four values of an array, at any address that its elements have.
template <typename T>
using Four = T __attribute__((ext_vector_type(4), aligned(sizeof(T))));

// kFull: all four are inside the array.
template <bool kFull, typename T>
__device__ __forceinline__ Four<T> load4(const void* p, int64_t i, int64_t count) {
  const T* const at = static_cast<const T*>(p) + i;
  if constexpr (kFull) return *reinterpret_cast<const Four<T>*>(at);
  Four<T> v;
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = i + k < count ? at[k] : static_cast<T>(0);
  return v;
}

template <bool kFull, typename T>
__device__ __forceinline__ void store4(void* p, int64_t i, int64_t count, Four<T> v) {
  T* const at = static_cast<T*>(p) + i;
  if constexpr (kFull) {
    *reinterpret_cast<Four<T>*>(at) = v;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < count) at[k] = v[k];
  }
}

// Largest of the wave's values, as bits (non-negative floats, infinities and
// NaN order like their bits); NaN where that is not finite, so that a block which
// has met an infinity stands for NaN throughout, whatever its codes.  By rotations
// within rows of 16 lanes, then across them, on the vector ALU.
__device__ __forceinline__ float wave_max(float v) {
  int b = __builtin_bit_cast(int, v);
  auto step = [&](auto control) {
    const int o = __builtin_amdgcn_update_dpp(0, b, decltype(control)::value, 0xf, 0xf, true);
    b = static_cast<int>(max(static_cast<uint32_t>(b), static_cast<uint32_t>(o)));
  };
  step(std::integral_constant<int, 0x121>{});  // row_ror:1
  step(std::integral_constant<int, 0x122>{});
  step(std::integral_constant<int, 0x124>{});
  step(std::integral_constant<int, 0x128>{});
  uint32_t m = 0;
#pragma unroll
  for (int row = 0; row < 4; ++row)
    m = max(m, static_cast<uint32_t>(__builtin_amdgcn_readlane(b, 16 * row)));
  return __builtin_bit_cast(float, m < 0x7f800000u ? m : 0x7fc00000u);
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
// Codes of a block whose largest value is s.
//
// x / s, rounded once: with y = 1 / s rounded once, q = x y and the exact
// remainder x - q s give it as q + y (x - q s) (Markstein's theorem), three
// operations for each value instead of a division's ten.  The remainder is exact
// while s is at least 2^-60: a quotient that leads to a code other than 0 is
// above 2^-37, so x is above 2^-97 and the remainder a multiple of 2^-145.
// Other scales (0, NaN and the largest among them) divide.
//
// The root: the hardware's is within a unit in the last place, so the scaled root
// is within 1e-4 of the exact one, and only a value that close to halfway between
// two codes needs the root that is rounded once.
//
// With a division and three exact roots for every value, and a branch around each,
// the vector ALU bound the 8-bit step: 134 M values with the values' pass 790 us;
// so, with whole blocks apart from ends, 664 (3.23 GB, 4.9 TB/s, a copy's rate).
__device__ __forceinline__ void ratios(const float (&x)[4], float s, float (&r)[4]) {
  if (s >= 0x1p-60f && s <= 0x1p100f) {
    const float y = 1.0f / s;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float q = x[k] * y;
      r[k] = __builtin_fmaf(__builtin_fmaf(-q, s, x[k]), y, q);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = s > 0.0f ? x[k] / s : 0.0f;
  }
}

constexpr float kNearHalf = 0.5f - 1e-4f;

__device__ __forceinline__ Four<int8_t> encode_m(const float (&m)[4], float s) {
  float x[4], r[4], c[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = __builtin_fabsf(m[k]);
  ratios(x, s, r);
  bool near = false;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float t = __builtin_amdgcn_sqrtf(r[k]) * 127.0f;
    c[k] = __builtin_rintf(t);
    near |= __builtin_fabsf(t - c[k]) > kNearHalf;
  }
  if (near) {
#pragma unroll
    for (int k = 0; k < 4; ++k) c[k] = __builtin_rintf(__builtin_sqrtf(r[k]) * 127.0f);
  }
  Four<int8_t> out;
#pragma unroll
  for (int k = 0; k < 4; ++k) out[k] = static_cast<int8_t>(__builtin_copysignf(c[k], m[k]));
  return out;
}

__device__ __forceinline__ Four<uint8_t> encode_v(const float (&v)[4], float s) {
  float r[4], c[4];
  ratios(v, s, r);
  bool near = false;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float t = __builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(r[k])) * 255.0f;
    c[k] = __builtin_rintf(t);
    near |= __builtin_fabsf(t - c[k]) > kNearHalf;
  }
  if (near) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      c[k] = __builtin_rintf(__builtin_sqrtf(__builtin_sqrtf(r[k])) * 255.0f);
  }
  Four<uint8_t> out;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    out[k] = static_cast<uint8_t>(v[k] > 0.0f ? __builtin_fmaxf(c[k], 1.0f) : c[k]);
  return out;
}

// What a lane reads of a block: four values of each array, states as they lie.
template <int kBits, bool kFull, typename G>
struct Loaded {
  typedef typename std::conditional<kBits == 8, int8_t, float>::type M;
  typedef typename std::conditional<kBits == 8, uint8_t, float>::type V;
  Four<float> p;
  Four<G> g;
  Four<M> m;
  Four<V> v;
  float ms, vs;

  __device__ __forceinline__ void read(const Entry& e, int64_t block) {
    const int64_t i = block * kWaveValues + (threadIdx.x & 63) * 4;
    p = load4<kFull, float>(e.p, i, e.count);
    g = load4<kFull, G>(e.g, i, e.count);
    m = load4<kFull, M>(e.m, i, e.count);
    v = load4<kFull, V>(e.v, i, e.count);
    if constexpr (kBits == 8) ms = e.ms[block], vs = e.vs[block];
  }

  // The step, and what it writes.  Values past the tensor's end read as zeros,
  // which a block's largest does not see.
  __device__ __forceinline__ void step(const Entry& e, const AdamwHyper& h, int64_t block) {
    const int64_t i = block * kWaveValues + (threadIdx.x & 63) * 4;
    float m1[4], v1[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float gk = static_cast<float>(g[k]) * h.grad_scale;
      float m0, v0;
      if constexpr (kBits == 8) m0 = decode_m(m[k], ms), v0 = decode_v(v[k], vs);
      else m0 = m[k], v0 = v[k];
      m1[k] = h.beta1 * m0 + h.rest1 * gk;
      v1[k] = h.beta2 * v0 + h.rest2 * (gk * gk);
      const float u = m1[k] / (__builtin_sqrtf(v1[k]) * h.root + h.eps);
      p[k] = p[k] * e.keep - h.step_size * u;
    }
    store4<kFull, float>(e.p, i, e.count, p);
    if constexpr (kBits == 8) {
      ms = wave_max(largest4(m1));
      vs = wave_max(largest4(v1));
      if ((threadIdx.x & 63) == 0) e.ms[block] = ms, e.vs[block] = vs;
      m = encode_m(m1, ms);
      v = encode_v(v1, vs);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) m[k] = m1[k], v[k] = v1[k];
    }
    store4<kFull, M>(e.m, i, e.count, m);
    store4<kFull, V>(e.v, i, e.count, v);
  }
};

// This wave's blocks of its workgroup's chunk: the first, and how many there are,
// the last of which may be shorter than 256 values.
__device__ __forceinline__ int wave_blocks(const Entry& e, int64_t& first) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  first = (static_cast<int64_t>(blockIdx.x - e.first) * (kThreads / 64) + wave) * kWaveBlocks;
  const int64_t left = (e.count + kWaveValues - 1) / kWaveValues - first;
  return static_cast<int>(min<int64_t>(max<int64_t>(left, 0), kWaveBlocks));
}

// Where the wave has all its blocks whole it reads two before it steps either.  HBM
// bounds it: 201 M values with 32-bit states and bfloat16 gradients 968 us (5.24 GB,
// 5.4 TB/s), one value a lane and access 2190; 8 bits: above.
template <int kBits, typename G>
__global__ __launch_bounds__(kThreads) void adamw_kernel(Args a) {
  const Entry& e = a.e[entry_of(a, blockIdx.x)];
  int64_t first;
  const int blocks = wave_blocks(e, first);
  if ((first + kWaveBlocks) * kWaveValues <= e.count) {
#pragma unroll 1
    for (int64_t b = first; b < first + kWaveBlocks; b += 2) {
      Loaded<kBits, true, G> x, y;
      x.read(e, b);
      y.read(e, b + 1);
      x.step(e, a.h, b);
      y.step(e, a.h, b + 1);
    }
  } else {
#pragma unroll 1
    for (int64_t b = first; b < first + blocks; ++b) {
      Loaded<kBits, false, G> x;
      x.read(e, b);
      x.step(e, a.h, b);
    }
  }
}

// What 8-bit states stand for, written where an entry's p and g point.
template <bool kFull>
__device__ __forceinline__ void values_block(const Entry& e, int64_t b) {
  const int64_t i = b * kWaveValues + (threadIdx.x & 63) * 4;
  const Four<int8_t> m = load4<kFull, int8_t>(e.m, i, e.count);
  const Four<uint8_t> v = load4<kFull, uint8_t>(e.v, i, e.count);
  const float ms = e.ms[b], vs = e.vs[b];
  Four<float> mo, vo;
#pragma unroll
  for (int k = 0; k < 4; ++k) mo[k] = decode_m(m[k], ms), vo[k] = decode_v(v[k], vs);
  store4<kFull, float>(e.p, i, e.count, mo);
  store4<kFull, float>(const_cast<void*>(e.g), i, e.count, vo);
}

__global__ __launch_bounds__(kThreads) void values_kernel(Args a) {
  const Entry& e = a.e[entry_of(a, blockIdx.x)];
  int64_t first;
  const int blocks = wave_blocks(e, first);
  if ((first + kWaveBlocks) * kWaveValues <= e.count) {
#pragma unroll
    for (int b = 0; b < kWaveBlocks; ++b) values_block<true>(e, first + b);
  } else {
    for (int b = 0; b < blocks; ++b) values_block<false>(e, first + b);
  }
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
        auto launch = [&](auto kernel) {
          hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a);
        };
        if (state_bits == 8) {
          if (grad_dtype == kF32) launch(adamw_kernel<8, float>);
          else if (grad_dtype == kF16) launch(adamw_kernel<8, _Float16>);
          else launch(adamw_kernel<8, __bf16>);
        } else {
          if (grad_dtype == kF32) launch(adamw_kernel<32, float>);
          else if (grad_dtype == kF16) launch(adamw_kernel<32, _Float16>);
          else launch(adamw_kernel<32, __bf16>);
        }
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
