// The gated linear layer and its gradients (gfx950):
//   G = X Wg + bg, U = X Wu + bu, Y = act(G) U;
//   dU = dY act(G), dG = dY U act'(G), and the gradients of two linear layers.
#include <algorithm>

#include "activation.h"
#include "layers.h"

namespace sgc {
namespace {

constexpr int kThreads = 256;

struct CombineArgs {
  int64_t M, N;
  int activation;
  const float *g, *u;
  int64_t ldg, ldu;
  float* y;
  int64_t ldy;
};
__global__ __launch_bounds__(kThreads) void combine_kernel(CombineArgs a) {
  const int64_t j = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (j >= a.N) return;
  for (int64_t i = blockIdx.y; i < a.M; i += gridDim.y)
    a.y[i * a.ldy + j] = activate(a.activation, a.g[i * a.ldg + j]) * a.u[i * a.ldu + j];
}

__global__ __launch_bounds__(kThreads) void gate_grad_kernel(GatedGradArgs a, float* dg, float* du) {
  const int64_t j = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (j >= a.N) return;
  for (int64_t i = blockIdx.y; i < a.M; i += gridDim.y) {
    const float dy = a.dy[i * a.lddy + j], g = a.z[0][i * a.ldz[0] + j];
    const float u = a.z[1][i * a.ldz[1] + j];
    dg[i * a.N + j] = dy * u * activate_grad(a.activation, g);
    du[i * a.N + j] = dy * activate(a.activation, g);
  }
}

dim3 grid_of(int64_t M, int64_t N) {
  return dim3(static_cast<unsigned>((N + kThreads - 1) / kThreads),
              static_cast<unsigned>(std::min<int64_t>(M, 65535)));
}

int64_t matrix_bytes(int64_t M, int64_t N) { return round_up(4 * M * N, 256); }

}  // namespace

size_t gated_ws(int64_t M, int64_t N, int64_t K) {
  if (M == 0 || N == 0) return 0;
  return static_cast<size_t>(2 * matrix_bytes(M, N)) + linear_ws(M, N, K);
}

hipError_t launch_gated(const GatedArgs& a, void* ws, hipStream_t stream) {
  char* const base = static_cast<char*>(ws);
  void* const linear = base + 2 * matrix_bytes(a.M, a.N);
  float* z[2];
  int64_t ldz[2];
  for (int i = 0; i < 2; ++i) {
    z[i] = a.z[i] ? a.z[i] : reinterpret_cast<float*>(base + i * matrix_bytes(a.M, a.N));
    ldz[i] = a.z[i] ? a.ldz[i] : a.N;
    LinearArgs l{};
    l.M = a.M, l.N = a.N, l.K = a.K;
    l.x = a.x, l.ldx = a.ldx;
    l.w = a.w[i], l.ldw = a.ldw[i], l.transpose_w = a.transpose_w;
    l.e.bias = a.bias[i];
    l.y = z[i], l.ldy = ldz[i];
    l.scale = a.scale, l.variant = a.variant;
    const hipError_t err = launch_linear(l, linear, stream);
    if (err != hipSuccess) return err;
  }
  const CombineArgs c{a.M, a.N, a.activation, z[0], z[1], ldz[0], ldz[1], a.y, a.ldy};
  hipLaunchKernelGGL(combine_kernel, grid_of(a.M, a.N), dim3(kThreads), 0, stream, c);
  return hipGetLastError();
}

size_t gated_grad_ws(int64_t M, int64_t N, int64_t K) {
  if (M == 0 || N == 0) return 0;
  return static_cast<size_t>(2 * matrix_bytes(M, N)) + linear_grad_ws(M, N, K);
}

hipError_t launch_gated_grad(const GatedGradArgs& a, void* ws, hipStream_t stream) {
  char* const base = static_cast<char*>(ws);
  float* d[2] = {reinterpret_cast<float*>(base),
                 reinterpret_cast<float*>(base + matrix_bytes(a.M, a.N))};
  if (a.M > 0 && a.N > 0) {
    hipLaunchKernelGGL(gate_grad_kernel, grid_of(a.M, a.N), dim3(kThreads), 0, stream, a, d[0],
                       d[1]);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  for (int i = 0; i < 2; ++i) {
    LinearGradArgs l{};
    l.M = a.M, l.N = a.N, l.K = a.K;
    l.dy = d[i], l.lddy = a.N;
    l.x = a.x, l.ldx = a.ldx;
    l.w = a.w[i], l.ldw = a.ldw[i], l.transpose_w = a.transpose_w;
    l.dx = a.dx, l.lddx = a.lddx, l.add_dx = i > 0;
    l.dw = a.dw[i], l.lddw = a.lddw[i], l.dbias = a.dbias[i];
    l.scale = a.scale, l.variant = a.variant;
    const hipError_t err = launch_linear_grad(l, base + 2 * matrix_bytes(a.M, a.N), stream);
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace sgc
