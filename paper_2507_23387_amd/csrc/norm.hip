// Layer norm of rows and its gradients (gfx950).
//
// Forward, per row: mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps),
// y = (x - mu) r w + b.  The variance is formed from the centred values, so a
// row whose mean is large against its spread keeps its digits.
// Backward, with h = (x - mu) r and g = dy w, per row:
// dx = r (g - mean(g) - h mean(g h)); over the rows: dw = sum dy h, db = sum dy.
// All sums are FP32 and have an order that the sizes alone fix.
#include <algorithm>
#include <atomic>

#include "gemm_common.h"
#include "layers.h"

namespace sgc {
namespace {

// Element types and the 16-byte pieces that rows are read and written in, at any
// address that elements have.
template <int kDtype>
struct Elem;
template <>
struct Elem<kF32> {
  typedef float T;
  static constexpr int kE = 4;
  typedef float Piece __attribute__((ext_vector_type(4), aligned(4)));
};
template <>
struct Elem<kF16> {
  typedef _Float16 T;
  static constexpr int kE = 8;
  typedef _Float16 Piece __attribute__((ext_vector_type(8), aligned(2)));
};
template <>
struct Elem<kBF16> {
  typedef __bf16 T;
  static constexpr int kE = 8;
  typedef __bf16 Piece __attribute__((ext_vector_type(8), aligned(2)));
};

constexpr int kThreads = 256;

// Elements j .. j + kE - 1 of a row of n, zeros past its end.
template <int kDtype>
__device__ __forceinline__ void load_piece(const typename Elem<kDtype>::T* row, int j, int n,
                                           float* v) {
  using L = Elem<kDtype>;
  if (j + L::kE <= n) {
    const typename L::Piece p = *reinterpret_cast<const typename L::Piece*>(row + j);
#pragma unroll
    for (int e = 0; e < L::kE; ++e) v[e] = static_cast<float>(p[e]);
  } else {
#pragma unroll
    for (int e = 0; e < L::kE; ++e) v[e] = j + e < n ? static_cast<float>(row[j + e]) : 0.0f;
  }
}

template <int kDtype>
__device__ __forceinline__ void store_piece(typename Elem<kDtype>::T* row, int j, int n,
                                            const float* v) {
  using L = Elem<kDtype>;
  if (j + L::kE <= n) {
    typename L::Piece p;
#pragma unroll
    for (int e = 0; e < L::kE; ++e) p[e] = static_cast<typename L::T>(v[e]);
    *reinterpret_cast<typename L::Piece*>(row + j) = p;
  } else {
#pragma unroll
    for (int e = 0; e < L::kE; ++e)
      if (j + e < n) row[j + e] = static_cast<typename L::T>(v[e]);
  }
}

// The kP values a thread of a row's kT holds: pieces t, t + kT, ... of the row.
template <int kDtype, int kT, int kP>
__device__ __forceinline__ void load_row(const typename Elem<kDtype>::T* row, int t, int n,
                                         float (&v)[kP]) {
  constexpr int kE = Elem<kDtype>::kE;
#pragma unroll
  for (int c = 0; c < kP / kE; ++c) load_piece<kDtype>(row, (c * kT + t) * kE, n, v + c * kE);
}

// The same pieces as they lie.
template <int kDtype, int kT, int kP>
__device__ __forceinline__ void load_raw(const typename Elem<kDtype>::T* row, int t, int n,
                                         typename Elem<kDtype>::Piece (&p)[kP / Elem<kDtype>::kE]) {
  using L = Elem<kDtype>;
#pragma unroll
  for (int c = 0; c < kP / L::kE; ++c) {
    const int j = (c * kT + t) * L::kE;
    if (j + L::kE <= n) {
      p[c] = *reinterpret_cast<const typename L::Piece*>(row + j);
    } else {
#pragma unroll
      for (int e = 0; e < L::kE; ++e)
        p[c][e] = j + e < n ? row[j + e] : static_cast<typename L::T>(0.0f);
    }
  }
}

// Values j .. j + kE - 1 of an FP32 vector, `fill` where there is no vector.
template <int kE>
__device__ __forceinline__ void vector_piece(const float* p, int j, int n, float fill, float* v) {
#pragma unroll
  for (int e = 0; e < kE; e += 4) {
    if (p) {
      load_piece<kF32>(p, j + e, n, v + e);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[e + i] = fill;
    }
  }
}

// A thread's kP values of an FP32 vector (load_row).
template <int kDtype, int kT, int kP>
__device__ __forceinline__ void load_vector(const float* p, int t, int n, float fill,
                                            float (&v)[kP]) {
  constexpr int kE = Elem<kDtype>::kE;
#pragma unroll
  for (int c = 0; c < kP / kE; ++c) vector_piece<kE>(p, (c * kT + t) * kE, n, fill, v + c * kE);
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// Sums of kN values over the kT threads of a row, in `lds` (kN floats per wave of
// the workgroup; a slot of its own for each of the sums between two barriers).
template <int kT, int kN>
__device__ __forceinline__ void row_sums(float (&v)[kN], float* lds) {
#pragma unroll
  for (int i = 0; i < kN; ++i) v[i] = wave_sum(v[i]);
  if constexpr (kT > 64) {
    const int wave = threadIdx.x >> 6, first = wave / (kT / 64) * (kT / 64);
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < kN; ++i) lds[wave * kN + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < kT / 64; ++w) s += lds[(first + w) * kN + i];
      v[i] = s;
    }
  }
}

// Rows whose values fit the registers of kT threads, kP each: one pass over HBM.
// A workgroup walks the rows with a stride, so that weight and bias are read once
// and the next row is on its way while this one is reduced.  HBM bounds it: 16384 x
// 4096 98 us in FP32 (5.5 TB/s), 46 in bfloat16 (5.8); three passes took 209.
template <int kDtype, int kT, int kP>
__global__ __launch_bounds__(kT < kThreads ? kThreads : kT, kP <= 8 ? 8 : 4) void norm_rows_kernel(
    NormArgs a) {
  typedef typename Elem<kDtype>::T T;
  constexpr int kE = Elem<kDtype>::kE, kBlock = kT < kThreads ? kThreads : kT, kRows = kBlock / kT;
  __shared__ float lds[2][kBlock / 64];
  const int t = threadIdx.x % kT, n = static_cast<int>(a.cols);
  float w[kP], b[kP], next[kP];
  load_vector<kDtype, kT, kP>(a.weight, t, n, 1.0f, w);
  load_vector<kDtype, kT, kP>(a.bias, t, n, 0.0f, b);
  const float rn = 1.0f / static_cast<float>(n);
  int64_t i = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / kT;
  const int64_t stride = static_cast<int64_t>(gridDim.x) * kRows;
  auto fetch = [&](int64_t row) {
    load_row<kDtype, kT, kP>(static_cast<const T*>(a.x) + min(row, a.rows - 1) * a.ldx, t, n, next);
  };
  fetch(i);
  // A workgroup's rows end together (kT > 64: one row; kT = 64: no barrier).
  for (; i < a.rows; i += stride) {
    float x[kP];
#pragma unroll
    for (int e = 0; e < kP; ++e) x[e] = next[e];
    // In place, the next row is read before this one is written.
    if (i + stride < a.rows) fetch(i + stride);
    float s[1] = {0.0f};
#pragma unroll
    for (int e = 0; e < kP; ++e) s[0] += x[e];
    row_sums<kT, 1>(s, lds[0]);
    // A division, so that a row of equal values whose sum is exact is centred to zeros.
    const float mu = s[0] / static_cast<float>(n);
    s[0] = 0.0f;
#pragma unroll
    for (int e = 0; e < kP; ++e) {
      x[e] -= mu;
      if ((e / kE * kT + t) * kE + e % kE < n) s[0] += x[e] * x[e];
    }
    row_sums<kT, 1>(s, lds[1]);
    const float r = 1.0f / __builtin_sqrtf(s[0] * rn + a.eps);
    T* const y = static_cast<T*>(a.y) + i * a.ldy;
#pragma unroll
    for (int c = 0; c < kP / kE; ++c) {
      float o[kE];
#pragma unroll
      for (int e = 0; e < kE; ++e) o[e] = x[c * kE + e] * r * w[c * kE + e] + b[c * kE + e];
      store_piece<kDtype>(y, (c * kT + t) * kE, n, o);
    }
    if (t == 0) {
      if (a.mean) a.mean[i] = mu;
      if (a.rstd) a.rstd[i] = r;
    }
  }
}

// Rows of any length: a workgroup of 1024 threads per row, three passes over it, the
// last two from the caches.  A thread at a value and 256 to a row, it was the wait for
// one load after the other: 64 x 33000 53 us, so 11; 4096 x 33000 530 and 280 (3.9 TB/s).
constexpr int kLongThreads = 1024;

// f(j, piece of x at j) over a row's pieces.
template <int kDtype, typename F>
__device__ __forceinline__ void each_piece(const typename Elem<kDtype>::T* row, int n, F f) {
  constexpr int kE = Elem<kDtype>::kE;
#pragma unroll 2
  for (int64_t j = threadIdx.x * kE; j < n; j += kLongThreads * kE) {
    float v[kE];
    load_piece<kDtype>(row, static_cast<int>(j), n, v);
    f(static_cast<int>(j), v);
  }
}

template <int kDtype>
__global__ __launch_bounds__(kLongThreads) void norm_kernel(NormArgs a) {
  typedef typename Elem<kDtype>::T T;
  constexpr int kE = Elem<kDtype>::kE;
  __shared__ float lds[2][kLongThreads / 64];
  const int n = static_cast<int>(a.cols);
  for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + i * a.ldx;
    T* y = static_cast<T*>(a.y) + i * a.ldy;
    float s[1] = {0.0f};
    each_piece<kDtype>(x, n, [&](int, const float (&v)[kE]) {
#pragma unroll
      for (int e = 0; e < kE; ++e) s[0] += v[e];
    });
    row_sums<kLongThreads, 1>(s, lds[0]);
    const float mu = s[0] / static_cast<float>(a.cols);
    s[0] = 0.0f;
    each_piece<kDtype>(x, n, [&](int j, const float (&v)[kE]) {
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const float d = j + e < n ? v[e] - mu : 0.0f;
        s[0] += d * d;
      }
    });
    row_sums<kLongThreads, 1>(s, lds[1]);
    const float r = 1.0f / __builtin_sqrtf(s[0] / static_cast<float>(a.cols) + a.eps);
    each_piece<kDtype>(x, n, [&](int j, const float (&v)[kE]) {
      float w[kE], b[kE], o[kE];
      vector_piece<kE>(a.weight, j, n, 1.0f, w);
      vector_piece<kE>(a.bias, j, n, 0.0f, b);
#pragma unroll
      for (int e = 0; e < kE; ++e) o[e] = (v[e] - mu) * r * w[e] + b[e];
      store_piece<kDtype>(y, j, n, o);
    });
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[i] = mu;
      if (a.rstd) a.rstd[i] = r;
    }
  }
}

// Gradients of rows whose values fit the registers of kT threads, kP each: dX, and
// the column sums of the workgroup's rows, in one pass over HBM.  1024 threads
// work on 1024 / kT rows at a time, each with the columns of its values; at the
// end those threads' sums are added in LDS, row by row of threads, and the
// workgroup writes one slab of partial sums.  16384 x 4096: 152 us in FP32 (5.3 TB/s),
// 78 in bfloat16 (5.2 TB/s); dX and the sums in passes of their own took 315 there.
constexpr int kGradThreads = 1024;

template <int kDtype, int kT, int kP>
__global__ __launch_bounds__(kGradThreads) void norm_grad_rows_kernel(NormGradArgs a) {
  typedef typename Elem<kDtype>::T T;
  constexpr int kE = Elem<kDtype>::kE, kRows = kGradThreads / kT;
  // The next row is on its way, as it lies, while one is reduced, but not at 16 values
  // a thread, where its registers spill.  A second one gives nothing: 16384 x 4096 in FP32
  // 156 us, so 152; calls in bfloat16 87.4, so 86.5, of 32000 x 500 31.5 and 31.4.
  constexpr bool kAhead = kP <= 8;
  __shared__ float lds[2][2 * kGradThreads / 64];
  extern __shared__ float sums[];  // 2 x kT x kP
  static_assert(2 * kT * kP * sizeof(float) <= 128 * 1024, "the sums fit LDS");
  const int t = threadIdx.x % kT, group = threadIdx.x / kT, n = static_cast<int>(a.cols);
  float w[kP], dw[kP], db[kP];
  load_vector<kDtype, kT, kP>(a.weight, t, n, 1.0f, w);
#pragma unroll
  for (int e = 0; e < kP; ++e) dw[e] = db[e] = 0.0f;
  const float rn = 1.0f / static_cast<float>(n);
  const int64_t stride = static_cast<int64_t>(gridDim.x) * kRows;
  int64_t first = static_cast<int64_t>(blockIdx.x) * kRows;
  struct Ahead {
    typename Elem<kDtype>::Piece x[kP / kE], g[kP / kE];
    float mu, r;
  };
  auto fetch = [&](int64_t row, Ahead& to) {
    row = min(row + group, a.rows - 1);
    load_raw<kDtype, kT, kP>(static_cast<const T*>(a.x) + row * a.ldx, t, n, to.x);
    load_raw<kDtype, kT, kP>(static_cast<const T*>(a.dy) + row * a.lddy, t, n, to.g);
    to.mu = a.mean[row];
    to.r = a.rstd[row];
  };
  // The whole workgroup takes every step (the sums wait at barriers); threads past
  // the last row repeat it and keep nothing.
  auto step = [&](Ahead& in, float* slot) {
    const bool mine = first + group < a.rows;
    const float mu = in.mu, r = in.r;
    float h[kP], g[kP], s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < kP; ++e) {
      const bool inside = (e / kE * kT + t) * kE + e % kE < n;
      const float dy = static_cast<float>(in.g[e / kE][e % kE]);
      h[e] = inside ? (static_cast<float>(in.x[e / kE][e % kE]) - mu) * r : 0.0f;
      dw[e] += mine ? dy * h[e] : 0.0f;
      db[e] += mine ? dy : 0.0f;
      g[e] = dy * w[e];
      s[0] += g[e];
      s[1] += g[e] * h[e];
    }
    if (kAhead && first + stride < a.rows) fetch(first + stride, in);
    row_sums<kT, 2>(s, slot);
    if (mine) {
      const float m1 = s[0] * rn, m2 = s[1] * rn;
      T* const dx = static_cast<T*>(a.dx) + (first + group) * a.lddx;
#pragma unroll
      for (int c = 0; c < kP / kE; ++c) {
        float o[kE];
#pragma unroll
        for (int e = 0; e < kE; ++e) o[e] = r * (g[c * kE + e] - m1 - h[c * kE + e] * m2);
        store_piece<kDtype>(dx, (c * kT + t) * kE, n, o);
      }
    }
    first += stride;
  };
  Ahead in;
  if (kAhead) fetch(first, in);
  for (int turn = 0; first < a.rows; turn ^= 1) {
    if (!kAhead) fetch(first, in);
    step(in, lds[turn]);
  }
  if (!a.dweight && !a.dbias) return;
  // Value e of thread t at e * kT + t: neighbours in neighbouring banks.
  for (int q = 0; q < kRows; ++q) {
    if (group == q) {
#pragma unroll
      for (int e = 0; e < kP; ++e) {
        const int at = e * kT + t;
        sums[at] = q ? sums[at] + dw[e] : dw[e];
        sums[kT * kP + at] = q ? sums[kT * kP + at] + db[e] : db[e];
      }
    }
    __syncthreads();
  }
  float* const out = a.partial + static_cast<int64_t>(blockIdx.x) * 2 * a.cols;
  for (int j = threadIdx.x; j < n; j += kGradThreads) {
    const int piece = j / kE, at = (piece / kT * kE + j % kE) * kT + piece % kT;
    out[j] = sums[at];
    out[n + j] = sums[kT * kP + at];
  }
}

// dX of rows of any length, a workgroup per row.
template <int kDtype>
__global__ __launch_bounds__(kLongThreads) void norm_dx_kernel(NormGradArgs a) {
  typedef typename Elem<kDtype>::T T;
  constexpr int kE = Elem<kDtype>::kE;
  __shared__ float lds[2][2 * kLongThreads / 64];
  const int n = static_cast<int>(a.cols);
  int turn = 0;
  for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x, turn ^= 1) {
    const T* x = static_cast<const T*>(a.x) + i * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + i * a.lddy;
    T* dx = static_cast<T*>(a.dx) + i * a.lddx;
    const float mu = a.mean[i], r = a.rstd[i];
    // g = dY weight and h of a piece; zeros past the row's end.
    auto both = [&](int j, const float (&v)[kE], float (&g)[kE], float (&h)[kE]) {
      float w[kE];
      vector_piece<kE>(a.weight, j, n, 1.0f, w);
      load_piece<kDtype>(dy, j, n, g);
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        g[e] *= w[e];
        h[e] = j + e < n ? (v[e] - mu) * r : 0.0f;
      }
    };
    float s[2] = {0.0f, 0.0f};
    each_piece<kDtype>(x, n, [&](int j, const float (&v)[kE]) {
      float g[kE], h[kE];
      both(j, v, g, h);
#pragma unroll
      for (int e = 0; e < kE; ++e) s[0] += g[e], s[1] += g[e] * h[e];
    });
    row_sums<kLongThreads, 2>(s, lds[turn]);
    const float m1 = s[0] / static_cast<float>(a.cols), m2 = s[1] / static_cast<float>(a.cols);
    each_piece<kDtype>(x, n, [&](int j, const float (&v)[kE]) {
      float g[kE], h[kE], o[kE];
      both(j, v, g, h);
#pragma unroll
      for (int e = 0; e < kE; ++e) o[e] = r * (g[e] - m1 - h[e] * m2);
      store_piece<kDtype>(dx, j, n, o);
    });
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

// Joins the slabs: a workgroup has 32 columns, every eighth slab a thread.
constexpr int kJoinCols = 32;
__global__ __launch_bounds__(kThreads) void norm_join_kernel(const float* __restrict__ partial,
                                                             int64_t slabs, int64_t cols,
                                                             float* dweight, float* dbias) {
  __shared__ float part[2][kThreads / kJoinCols][kJoinCols];
  const int c = threadIdx.x % kJoinCols, g = threadIdx.x / kJoinCols;
  const int64_t j = static_cast<int64_t>(blockIdx.x) * kJoinCols + c;
  float dw = 0.0f, db = 0.0f;
  if (j < cols) {
#pragma unroll 4
    for (int64_t s = g; s < slabs; s += kThreads / kJoinCols) {
      dw += partial[2 * s * cols + j];
      db += partial[(2 * s + 1) * cols + j];
    }
  }
  part[0][g][c] = dw;
  part[1][g][c] = db;
  __syncthreads();
  if (g != 0 || j >= cols) return;
#pragma unroll
  for (int q = 1; q < kThreads / kJoinCols; ++q) dw += part[0][q][c], db += part[1][q][c];
  if (dweight) dweight[j] = dw;
  if (dbias) dbias[j] = db;
}

unsigned row_grid(int64_t rows) {
  return static_cast<unsigned>(std::min<int64_t>(rows, int64_t{1} << 20));
}

template <int kDtype, int kT, int kP>
hipError_t forward_rows(const NormArgs& a, hipStream_t stream) {
  constexpr int kBlock = kT < kThreads ? kThreads : kT, kRows = kBlock / kT;
  // As many workgroups as run together (the registers of kP = 16 leave room for
  // 5 waves per SIMD).
  constexpr int kTogether = kP <= 8 ? 2048 / kBlock : kBlock == 1024 ? 1 : 1280 / kBlock;
  const int64_t grid = std::min<int64_t>((a.rows + kRows - 1) / kRows, 256 * kTogether);
  hipLaunchKernelGGL((norm_rows_kernel<kDtype, kT, kP>), dim3(static_cast<unsigned>(grid)),
                     dim3(kBlock), 0, stream, a);
  return hipGetLastError();
}

template <int kDtype>
hipError_t forward(const NormArgs& a, hipStream_t stream) {
  const int64_t n = a.cols;
  if (n > 0 && n <= 64 * 8) return forward_rows<kDtype, 64, 8>(a, stream);
  if (n > 0 && n <= 64 * 16) return forward_rows<kDtype, 64, 16>(a, stream);
  if (n > 0 && n <= 256 * 8) return forward_rows<kDtype, 256, 8>(a, stream);
  if (n > 0 && n <= 256 * 16) return forward_rows<kDtype, 256, 16>(a, stream);
  if (n > 0 && n <= 1024 * 8) return forward_rows<kDtype, 1024, 8>(a, stream);
  if (n > 0 && n <= 1024 * 16) return forward_rows<kDtype, 1024, 16>(a, stream);
  hipLaunchKernelGGL(norm_kernel<kDtype>, dim3(row_grid(a.rows)), dim3(kLongThreads), 0, stream, a);
  return hipGetLastError();
}

// Threads per row of the gradient's kernel, 0 where a row does not fit registers.
int grad_threads(int64_t cols) {
  for (int t = 64; t < 1024; t *= 2)
    if (cols <= t * 8) return t;
  return cols <= 1024 * 16 ? 1024 : 0;
}

hipError_t join(const NormGradArgs& a, int64_t slabs, hipStream_t stream) {
  if (!a.dweight && !a.dbias) return hipSuccess;
  const unsigned strips = static_cast<unsigned>((a.cols + kJoinCols - 1) / kJoinCols);
  hipLaunchKernelGGL(norm_join_kernel, dim3(strips), dim3(kThreads), 0, stream, a.partial, slabs,
                     a.cols, a.dweight, a.dbias);
  return hipGetLastError();
}

template <int kDtype, int kT, int kP>
hipError_t grad_rows(const NormGradArgs& a, hipStream_t stream) {
  constexpr size_t kLds = 2 * kT * kP * sizeof(float);
  static std::atomic<bool> done[kMaxDevices];
  const hipError_t attr = set_lds(&norm_grad_rows_kernel<kDtype, kT, kP>, kLds, done);
  if (attr != hipSuccess) return attr;
  const int64_t slabs = norm_slabs(a.rows, a.cols);
  hipLaunchKernelGGL((norm_grad_rows_kernel<kDtype, kT, kP>), dim3(static_cast<unsigned>(slabs)),
                     dim3(kGradThreads), kLds, stream, a);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  return join(a, slabs, stream);
}

template <int kDtype>
hipError_t grad(const NormGradArgs& a, hipStream_t stream) {
  if (a.rows == 0) return join(a, 0, stream);
  switch (grad_threads(a.cols)) {
    case 64: return grad_rows<kDtype, 64, 8>(a, stream);
    case 128: return grad_rows<kDtype, 128, 8>(a, stream);
    case 256: return grad_rows<kDtype, 256, 8>(a, stream);
    case 512: return grad_rows<kDtype, 512, 8>(a, stream);
    case 1024:
      return a.cols <= 1024 * 8 ? grad_rows<kDtype, 1024, 8>(a, stream)
                                : grad_rows<kDtype, 1024, 16>(a, stream);
    default: break;
  }
  // Longer rows.  The column sums first: dX may be dY.
  const int64_t slabs = norm_slabs(a.rows, a.cols);
  if (a.dweight || a.dbias) {
    const unsigned strips = static_cast<unsigned>((a.cols + kThreads - 1) / kThreads);
    hipLaunchKernelGGL(norm_dw_kernel<kDtype>, dim3(strips, static_cast<unsigned>(slabs)),
                       dim3(kThreads), 0, stream, a, (a.rows + slabs - 1) / slabs);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (const hipError_t e = join(a, slabs, stream); e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(norm_dx_kernel<kDtype>, dim3(row_grid(a.rows)), dim3(kLongThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

// One slab for each workgroup of the gradient's kernel, one per compute unit.
int64_t norm_slabs(int64_t rows, int64_t cols) {
  const int threads = grad_threads(cols);
  const int64_t at_a_time = threads ? kGradThreads / threads : 1;
  return std::min<int64_t>((rows + at_a_time - 1) / at_a_time, 256);
}

hipError_t launch_norm(const NormArgs& a, int dtype, hipStream_t stream) {
  switch (dtype) {
    case kF32: return forward<kF32>(a, stream);
    case kF16: return forward<kF16>(a, stream);
    case kBF16: return forward<kBF16>(a, stream);
    default: return hipErrorInvalidValue;
  }
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
