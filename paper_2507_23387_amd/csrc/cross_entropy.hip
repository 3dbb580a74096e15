// Cross entropy of a linear layer's rows over a vocabulary, and its gradients (gfx950).
//
// With z = X W + b: lse_i = log sum_j exp(z_ij), loss_i = lse_i - z_i,t.  The vocabulary
// is taken in pieces, of which no more than one piece's logits are in memory.  A row's
// maximum and sum of exponentials are kept for stretches of its columns and joined at
// the end, so that each logit is looked at once.
// Gradients, from g = dloss and h = dlse: D_ij = exp(z_ij - lse_i) (g_i + h_i) -
// [j = t_i] g_i, whose products are those of a linear layer (linear.hip).
#include <algorithm>

#include "layers.h"

namespace sgc {
namespace {

constexpr int kThreads = 256;
typedef float floatx4_u __attribute__((ext_vector_type(4), aligned(4)));

// exp(x) on the hardware's exp2: off by (|x| + 2) 2^-24 of itself.
__device__ __forceinline__ float exp_of(float x) {
  return __builtin_amdgcn_exp2f(1.44269504f * x);
}

// Sums of exponentials: sum exp(z) = sum * exp(top).
struct Exps {
  float top, sum;
  // Without a finite entry (top = -inf) the sum is 0.  A NaN or +inf makes it NaN.
  __device__ __forceinline__ void join(const Exps& o) {
    const float t = __builtin_fmaxf(top, o.top);
    const float s = t == -__builtin_inff() ? sum + o.sum
                                           : sum * exp_of(top - t) + o.sum * exp_of(o.top - t);
    top = t;
    sum = s;
  }
};

__device__ __forceinline__ int64_t target_at(const Ids& ids, int64_t i) {
  return ids.bits == 32 ? static_cast<const int32_t*>(ids.p)[i]
                        : static_cast<const int64_t*>(ids.p)[i];
}

// What the rows of a piece's logits leave.
struct PieceArgs {
  int64_t M, cols, first;  // columns first .. first + cols - 1 of the vocabulary
  const float* z;          // M x cols
  Ids targets;
  Exps* exps;     // slots x M
  float* at;      // the target's logit
  int64_t slot0;  // of this piece's first stretch
  int64_t stretch;
};

// A stretch of one row a workgroup.
__global__ __launch_bounds__(kThreads) void exps_kernel(PieceArgs g) {
  __shared__ Exps part[kThreads / 64];
  const int64_t c0 = blockIdx.y * g.stretch, c1 = min(g.cols, c0 + g.stretch);
  for (int64_t i = blockIdx.x; i < g.M; i += gridDim.x) {
    const float* const row = g.z + i * g.cols;
    Exps e{-__builtin_inff(), 0.0f};
    for (int64_t j = c0 + 4 * threadIdx.x; j < c1; j += 4 * kThreads) {
      float v[4];
      if (j + 3 < c1) {
        const floatx4_u p = *reinterpret_cast<const floatx4_u*>(row + j);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = p[k];
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = j + k < c1 ? row[j + k] : -__builtin_inff();
      }
      Exps o{__builtin_fmaxf(__builtin_fmaxf(v[0], v[1]), __builtin_fmaxf(v[2], v[3])), 0.0f};
      const float base = o.top == -__builtin_inff() ? 0.0f : o.top;
#pragma unroll
      for (int k = 0; k < 4; ++k) o.sum += exp_of(v[k] - base);
      e.join(o);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) e.join(Exps{__shfl_xor(e.top, d), __shfl_xor(e.sum, d)});
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = e;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
      for (int w = 1; w < kThreads / 64; ++w) e.join(part[w]);
      g.exps[(g.slot0 + blockIdx.y) * g.M + i] = e;
      const int64_t t = target_at(g.targets, i) - g.first;
      if (t >= c0 && t < c1) g.at[i] = row[t];
    }
    __syncthreads();  // the sums are read before the next row's are written
  }
}

// The rows' results from `slots` stretches: 16 rows a workgroup, every 16th stretch a
// thread.
constexpr int kJoinRows = 16, kJoinGroups = kThreads / kJoinRows;
__global__ __launch_bounds__(kThreads) void xent_join_kernel(int64_t M, int64_t V, int64_t slots,
                                                             const Exps* exps, const float* at,
                                                             Ids targets, float* loss,
                                                             float* lse) {
  __shared__ Exps part[kJoinGroups][kJoinRows];
  const int r = threadIdx.x % kJoinRows, q = threadIdx.x / kJoinRows;
  for (int64_t i0 = static_cast<int64_t>(blockIdx.x) * kJoinRows; i0 < M;
       i0 += static_cast<int64_t>(gridDim.x) * kJoinRows) {
    const int64_t i = i0 + r;
    Exps e{-__builtin_inff(), 0.0f};
    if (i < M) {
#pragma unroll 4
      for (int64_t s = q; s < slots; s += kJoinGroups) e.join(exps[s * M + i]);
    }
    part[q][r] = e;
    __syncthreads();
    if (q == 0 && i < M) {
      for (int k = 1; k < kJoinGroups; ++k) e.join(part[k][r]);
      const float l = e.top + __builtin_logf(e.sum);
      const int64_t t = target_at(targets, i);
      lse[i] = l;
      loss[i] = t < 0 ? 0.0f : t >= V ? __builtin_nanf("") : l - at[i];
    }
    __syncthreads();  // the sums are read before the next rows' are written
  }
}

// Z, a piece's logits, becomes D.
struct GradArgs {
  int64_t M, cols, first, vocab;
  float* z;
  Ids targets;
  const float *dloss, *dlse, *lse;
};
__global__ __launch_bounds__(kThreads) void xent_grad_kernel(GradArgs g) {
  const int64_t j = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) * 4;
  if (j >= g.cols) return;
  for (int64_t i = blockIdx.y; i < g.M; i += gridDim.y) {
    const int64_t t = target_at(g.targets, i);
    const float d = t < 0 ? 0.0f : t >= g.vocab ? __builtin_nanf("") : g.dloss[i];
    const float c = g.dlse ? d + g.dlse[i] : d, l = g.lse[i];
    float* const at = g.z + i * g.cols + j;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (j + k >= g.cols) break;
      const float p = c == 0.0f ? 0.0f : exp_of(at[k] - l) * c;
      at[k] = g.first + j + k == t ? p - d : p;
    }
  }
}

// Columns of a piece: what keeps its logits within 256 MiB, whole tiles of 256 columns.
int64_t piece_cols(int64_t M, int64_t V) {
  const int64_t most = std::max<int64_t>(1, (int64_t{64} << 20) / std::max<int64_t>(M, 1) / 256);
  return std::min(V, most * 256);
}

// Columns of a row that one workgroup reduces: few rows are shared by more of them.
int64_t stretch_cols(int64_t M, int64_t cols) {
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(cols / 1024, 1024 / M));
  return round_up((cols + parts - 1) / parts, 4);
}

int64_t stretches(int64_t M, int64_t cols) {
  const int64_t s = stretch_cols(M, cols);
  return (cols + s - 1) / s;
}

// Workgroups that take rows in turn, within a grid of 2^32 threads.
unsigned rows_grid(int64_t workgroups) {
  return static_cast<unsigned>(std::min<int64_t>(workgroups, int64_t{1} << 20));
}

struct Carver {
  char* base;
  size_t used;
  template <typename T>
  T* take(int64_t bytes) {
    char* const at = base + used;
    used += static_cast<size_t>(round_up(bytes, 256));
    return reinterpret_cast<T*>(at);
  }
};

const float* piece_of(const XentArgs& a, int64_t first) {
  return a.w + (a.transpose_w ? first * a.ldw : first);
}

LinearArgs logits_of(const XentArgs& a, int64_t first, int64_t cols, float* z) {
  LinearArgs l{};
  l.M = a.M, l.N = cols, l.K = a.K;
  l.x = a.x, l.ldx = a.ldx;
  l.w = piece_of(a, first), l.ldw = a.ldw, l.transpose_w = a.transpose_w;
  l.e.bias = a.bias ? a.bias + first : nullptr;
  l.y = z, l.ldy = cols;
  l.scale = a.scale, l.variant = a.variant;
  return l;
}

struct Workspace {
  float* z;
  Exps* exps;
  float* at;
  void* linear;
  int64_t piece, slots;
  size_t bytes;
};

Workspace carve(void* ws, int64_t M, int64_t V, int64_t K) {
  Carver c{static_cast<char*>(ws), 0};
  Workspace w{};
  w.piece = piece_cols(M, V);
  const int64_t rest = V % w.piece;
  w.slots = V / w.piece * stretches(M, w.piece) + (rest ? stretches(M, rest) : 0);
  w.z = c.take<float>(4 * M * w.piece);
  w.exps = c.take<Exps>(8 * M * w.slots);
  w.at = c.take<float>(4 * M);
  // Of both widths: fewer columns may take another path.
  w.linear = c.take<void>(static_cast<int64_t>(
      std::max(linear_ws(M, w.piece, K), linear_ws(M, rest, K))));
  w.bytes = c.used;
  return w;
}

struct GradWorkspace {
  float* z;
  void* linear;
  int64_t piece;
  size_t bytes;
};

GradWorkspace carve_grad(void* ws, int64_t M, int64_t V, int64_t K) {
  Carver c{static_cast<char*>(ws), 0};
  GradWorkspace w{};
  w.piece = piece_cols(M, V);
  const int64_t rest = V % w.piece;
  w.z = c.take<float>(4 * M * w.piece);
  w.linear = c.take<void>(static_cast<int64_t>(
      std::max(std::max(linear_ws(M, w.piece, K), linear_ws(M, rest, K)),
               std::max(linear_grad_ws(M, w.piece, K), linear_grad_ws(M, rest, K)))));
  w.bytes = c.used;
  return w;
}

}  // namespace

size_t xent_ws(int64_t M, int64_t V, int64_t K) {
  return M > 0 && V > 0 ? carve(nullptr, M, V, K).bytes : 0;
}

hipError_t launch_xent(const XentArgs& a, float* loss, float* lse, void* ws, hipStream_t stream) {
  Workspace w{};
  if (a.V > 0) w = carve(ws, a.M, a.V, a.K);
  hipError_t err = hipSuccess;
  int64_t slot = 0;
  for (int64_t first = 0; first < a.V && err == hipSuccess; first += w.piece) {
    const int64_t cols = std::min(w.piece, a.V - first);
    err = launch_linear(logits_of(a, first, cols, w.z), w.linear, stream);
    if (err != hipSuccess) break;
    const PieceArgs g{a.M, cols, first, w.z, a.targets, w.exps, w.at, slot,
                      stretch_cols(a.M, cols)};
    const int64_t parts = stretches(a.M, cols);
    hipLaunchKernelGGL(exps_kernel, dim3(rows_grid(a.M), static_cast<unsigned>(parts)),
                       dim3(kThreads), 0, stream, g);
    err = hipGetLastError();
    slot += parts;
  }
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL(xent_join_kernel,
                     dim3(rows_grid((a.M + kJoinRows - 1) / kJoinRows)),
                     dim3(kThreads), 0, stream, a.M, a.V, slot, w.exps, w.at, a.targets, loss,
                     lse);
  return hipGetLastError();
}

size_t xent_grad_ws(int64_t M, int64_t V, int64_t K) {
  return M > 0 && V > 0 ? carve_grad(nullptr, M, V, K).bytes : 0;
}

hipError_t launch_xent_grad(const XentGradArgs& a, void* ws, hipStream_t stream) {
  const XentArgs& x = a.x;
  hipError_t err = hipSuccess;
  if (x.M == 0 || x.V == 0) {
    if (a.dx) err = launch_zero(x.M, x.K, a.dx, a.lddx, stream);
    if (err == hipSuccess && a.dw)
      err = launch_zero(x.transpose_w ? x.V : x.K, x.transpose_w ? x.K : x.V, a.dw, a.lddw, stream);
    if (err == hipSuccess && a.dbias) err = launch_zero(1, x.V, a.dbias, x.V, stream);
    return err;
  }
  const GradWorkspace w = carve_grad(ws, x.M, x.V, x.K);
  for (int64_t first = 0; first < x.V && err == hipSuccess; first += w.piece) {
    const int64_t cols = std::min(w.piece, x.V - first);
    err = launch_linear(logits_of(x, first, cols, w.z), w.linear, stream);
    if (err != hipSuccess) break;
    const GradArgs g{x.M, cols, first, x.V, w.z, x.targets, a.dloss, a.dlse, a.lse};
    hipLaunchKernelGGL(xent_grad_kernel,
                       dim3(static_cast<unsigned>((cols + 4 * kThreads - 1) / (4 * kThreads)),
                            static_cast<unsigned>(std::min<int64_t>(x.M, 65535))),
                       dim3(kThreads), 0, stream, g);
    err = hipGetLastError();
    if (err != hipSuccess) break;
    LinearGradArgs l{};
    l.M = x.M, l.N = cols, l.K = x.K;
    l.dy = w.z, l.lddy = cols;
    l.x = x.x, l.ldx = x.ldx;
    l.w = piece_of(x, first), l.ldw = x.ldw, l.transpose_w = x.transpose_w;
    l.dx = a.dx, l.lddx = a.lddx, l.add_dx = first > 0;
    l.dw = a.dw ? a.dw + (x.transpose_w ? first * a.lddw : first) : nullptr, l.lddw = a.lddw;
    l.dbias = a.dbias ? a.dbias + first : nullptr;
    l.scale = x.scale, l.variant = x.variant;
    err = launch_linear_grad(l, w.linear, stream);
  }
  return err;
}

}  // namespace sgc
