// C-ABI of the layers: argument validation, workspace, dispatch.  The
// interface and its conventions are documented in include/sgemm_cube_layers.h.
#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "layers.h"
#include "sgemm_cube_layers.h"
#include "validate.h"

namespace sgc {
namespace {

constexpr int kInvalid = SGEMM_CUBE_ERR_INVALID_VALUE;

int status_of(hipError_t e) { return e == hipSuccess ? SGEMM_CUBE_OK : SGEMM_CUBE_ERR_HIP; }

bool valid_dtype(int dtype) { return dtype >= SGEMM_CUBE_F32 && dtype <= SGEMM_CUBE_BF16; }

// A rows x cols matrix operand: leading dimension, pointer (aligned to its
// elements) and extent.
bool matrix_ok(int64_t rows, int64_t cols, const void* p, int64_t ld, uint64_t elem) {
  if (ld < (cols > 1 ? cols : 1) || !ld_ok(rows, ld)) return false;
  return rows == 0 || cols == 0 || (p && reinterpret_cast<uintptr_t>(p) % elem == 0);
}

// A vector operand that may be absent.
bool vector_ok(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

// One operand's bytes, for the overlap checks.
struct Span {
  const void* p;
  uint64_t bytes;
};

bool hits(const Span& out, std::initializer_list<Span> others) {
  for (const Span& o : others)
    if (out.p && o.p && overlap(out.p, out.bytes, o.p, o.bytes)) return true;
  return false;
}

bool workspace_ok(const void* ws, size_t ws_bytes, size_t need) {
  return ws_bytes >= need && (need == 0 || (ws && reinterpret_cast<uintptr_t>(ws) % 256 == 0));
}

// AdamW's list of tensors: 0 where every entry is valid.
int check_adamw_list(int64_t tensors, const sgemm_cube_adamw_tensor_t* list, int state_bits) {
  if (tensors < 0 || (tensors > 0 && !list)) return kInvalid;
  if (state_bits != 8 && state_bits != 32) return kInvalid;
  for (int64_t i = 0; i < tensors; ++i) {
    const sgemm_cube_adamw_tensor_t& t = list[i];
    if (t.count < 0) return kInvalid;
    if (t.count > kAdamwMaxCount) return SGEMM_CUBE_ERR_NOT_SUPPORTED;
    if (t.count == 0) continue;
    if (!t.exp_avg || !t.exp_avg_sq) return kInvalid;
    if (state_bits == 32 && !(vector_ok(t.exp_avg) && vector_ok(t.exp_avg_sq))) return kInvalid;
    if (state_bits == 8 && !(t.exp_avg_scale && t.exp_avg_sq_scale &&
                             vector_ok(t.exp_avg_scale) && vector_ok(t.exp_avg_sq_scale)))
      return kInvalid;
  }
  return SGEMM_CUBE_OK;
}

bool valid_activation(int a) { return a >= SGEMM_CUBE_ACT_NONE && a <= SGEMM_CUBE_ACT_SILU; }

// Limits of the kernels of an M x N x K product.
bool product_exceeds(int64_t M, int64_t N, int64_t K) {
  return M > kMaxDim || N > kMaxDim || K > kMaxDim || round_up_tiles_exceed(M, N);
}

size_t norm_grad_ws(int64_t rows, int64_t cols) {
  return static_cast<size_t>(round_up(norm_slabs(rows, cols) * 2 * cols * 4, 256));
}

}  // namespace
}  // namespace sgc

#pragma GCC visibility push(default)
extern "C" {

size_t sgemm_cube_linear_workspace_size(int64_t M, int64_t N, int64_t K) {
  if (M < 0 || N < 0 || K < 0 || sgc::product_exceeds(M, N, K)) return 0;
  return sgc::linear_ws(M, N, K);
}

int sgemm_cube_linear(int64_t M, int64_t N, int64_t K, const float* X, int64_t ldx,
                      const float* W, int64_t ldw, int transpose_w, const float* bias,
                      int activation, const float* R, int64_t ldr, float* Y, int64_t ldy,
                      float* Z, int64_t ldz, float scale, int accum_order, void* ws,
                      size_t ws_bytes, hipStream_t stream) {
  using namespace sgc;
  if (M < 0 || N < 0 || K < 0 || !valid_order(accum_order) || !valid_activation(activation) ||
      !valid_scale(scale))
    return kInvalid;
  const int64_t wr = transpose_w ? N : K, wc = transpose_w ? K : N;
  if (!matrix_ok(M, K, X, ldx, 4) || !matrix_ok(wr, wc, W, ldw, 4) || !vector_ok(bias) ||
      (R && !matrix_ok(M, N, R, ldr, 4)) || !matrix_ok(M, N, Y, ldy, 4) ||
      (Z && !matrix_ok(M, N, Z, ldz, 4)))
    return kInvalid;
  if (product_exceeds(M, N, K)) return SGEMM_CUBE_ERR_NOT_SUPPORTED;
  const size_t need = linear_ws(M, N, K);
  if (!workspace_ok(ws, ws_bytes, need)) return kInvalid;
  const Span x{X, span_bytes(M, K, ldx, 4)}, w{W, span_bytes(wr, wc, ldw, 4)};
  const Span b{bias, 4 * static_cast<uint64_t>(N)}, r{R, span_bytes(M, N, ldr, 4)};
  const Span y{Y, span_bytes(M, N, ldy, 4)}, z{Z, span_bytes(M, N, ldz, 4)}, wsp{ws, need};
  const bool in_place = R == Y && ldr == ldy;
  if (hits(y, {x, w, b, z, wsp}) || (!in_place && hits(y, {r})) || hits(z, {x, w, b, r, wsp}) ||
      hits(wsp, {x, w, b, r}))
    return kInvalid;
  if (M == 0 || N == 0) return SGEMM_CUBE_OK;
  LinearArgs a{M, N, K, X, ldx, W, ldw, transpose_w != 0, Epilogue{}, Y, ldy, scale,
               variant_of(accum_order)};
  a.e.bias = bias;
  a.e.activation = activation;
  a.e.r = R, a.e.ldr = ldr;
  a.e.z = Z, a.e.ldz = ldz;
  return status_of(launch_linear(a, ws, stream));
}

size_t sgemm_cube_linear_backward_workspace_size(int64_t M, int64_t N, int64_t K) {
  using namespace sgc;
  if (M < 0 || N < 0 || K < 0 || product_exceeds(M, K, N) || product_exceeds(K, N, M) ||
      product_exceeds(N, K, M))
    return 0;
  return linear_grad_ws(M, N, K);
}

int sgemm_cube_linear_backward(int64_t M, int64_t N, int64_t K, const float* dY, int64_t lddy,
                               const float* Z, int64_t ldz, const float* X, int64_t ldx,
                               const float* W, int64_t ldw, int transpose_w, int activation,
                               float* dX, int64_t lddx, float* dW, int64_t lddw, float* dbias,
                               float scale, int accum_order, void* ws, size_t ws_bytes,
                               hipStream_t stream) {
  using namespace sgc;
  if (M < 0 || N < 0 || K < 0 || !valid_order(accum_order) || !valid_activation(activation) ||
      !valid_scale(scale))
    return kInvalid;
  const int64_t wr = transpose_w ? N : K, wc = transpose_w ? K : N;
  const bool act = activation != SGEMM_CUBE_ACT_NONE;
  if (!matrix_ok(M, N, dY, lddy, 4) || (act && !matrix_ok(M, N, Z, ldz, 4)) ||
      !matrix_ok(M, K, X, ldx, 4) || !matrix_ok(wr, wc, W, ldw, 4) ||
      (dX && !matrix_ok(M, K, dX, lddx, 4)) || (dW && !matrix_ok(wr, wc, dW, lddw, 4)) ||
      !vector_ok(dbias))
    return kInvalid;
  if (product_exceeds(M, K, N) || product_exceeds(K, N, M) || product_exceeds(N, K, M))
    return SGEMM_CUBE_ERR_NOT_SUPPORTED;
  const size_t need = linear_grad_ws(M, N, K);
  if (!workspace_ok(ws, ws_bytes, need)) return kInvalid;
  if (!act) Z = nullptr;
  const Span dy{dY, span_bytes(M, N, lddy, 4)}, z{Z, span_bytes(M, N, ldz, 4)};
  const Span x{X, span_bytes(M, K, ldx, 4)}, w{W, span_bytes(wr, wc, ldw, 4)};
  const Span dx{dX, span_bytes(M, K, lddx, 4)}, dw{dW, span_bytes(wr, wc, lddw, 4)};
  const Span db{dbias, 4 * static_cast<uint64_t>(N)}, wsp{ws, need};
  if (hits(dx, {dy, z, x, w, dw, db, wsp}) || hits(dw, {dy, z, x, w, db, wsp}) ||
      hits(db, {dy, z, x, w, wsp}) || hits(wsp, {dy, z, x, w}))
    return kInvalid;
  const LinearGradArgs a{M, N, K, dY, lddy, Z, ldz, X, ldx, W, ldw, transpose_w != 0, activation,
                         dX, lddx, dW, lddw, dbias, scale, variant_of(accum_order)};
  return status_of(launch_linear_grad(a, ws, stream));
}

int sgemm_cube_layer_norm(int64_t rows, int64_t cols, int dtype, const void* X, int64_t ldx,
                          const float* weight, const float* bias, float eps, void* Y,
                          int64_t ldy, float* mean, float* rstd, hipStream_t stream) {
  using namespace sgc;
  if (rows < 0 || cols < 0 || !valid_dtype(dtype) || !(eps >= 0.0f) || std::isinf(eps))
    return kInvalid;
  const uint64_t elem = dtype_bytes(dtype);
  if (!matrix_ok(rows, cols, X, ldx, elem) || !matrix_ok(rows, cols, Y, ldy, elem) ||
      !vector_ok(weight) || !vector_ok(bias) || !vector_ok(mean) || !vector_ok(rstd))
    return kInvalid;
  const uint64_t r4 = 4 * static_cast<uint64_t>(rows), c4 = 4 * static_cast<uint64_t>(cols);
  const Span x{X, span_bytes(rows, cols, ldx, elem)}, y{Y, span_bytes(rows, cols, ldy, elem)};
  const Span w{weight, c4}, b{bias, c4}, mu{mean, r4}, rs{rstd, r4};
  const bool in_place = X == Y && ldx == ldy;
  if ((!in_place && hits(y, {x})) || hits(y, {w, b, mu, rs}) || hits(mu, {x, w, b, rs}) ||
      hits(rs, {x, w, b}))
    return kInvalid;
  if (rows > kMaxDim || cols > kMaxDim) return SGEMM_CUBE_ERR_NOT_SUPPORTED;
  if (rows == 0 || (cols == 0 && !mean && !rstd)) return SGEMM_CUBE_OK;
  const NormArgs a{rows, cols, X, ldx, weight, bias, eps, Y, ldy, mean, rstd};
  return status_of(launch_norm(a, dtype, stream));
}

size_t sgemm_cube_layer_norm_backward_workspace_size(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0 || rows > sgc::kMaxDim || cols > sgc::kMaxDim) return 0;
  return sgc::norm_grad_ws(rows, cols);
}

int sgemm_cube_layer_norm_backward(int64_t rows, int64_t cols, int dtype, const void* dY,
                                   int64_t lddy, const void* X, int64_t ldx, const float* weight,
                                   const float* mean, const float* rstd, void* dX, int64_t lddx,
                                   float* dweight, float* dbias, void* ws, size_t ws_bytes,
                                   hipStream_t stream) {
  using namespace sgc;
  if (rows < 0 || cols < 0 || !valid_dtype(dtype)) return kInvalid;
  const uint64_t elem = dtype_bytes(dtype);
  if (!matrix_ok(rows, cols, dY, lddy, elem) || !matrix_ok(rows, cols, X, ldx, elem) ||
      !matrix_ok(rows, cols, dX, lddx, elem) || !vector_ok(weight) || !vector_ok(mean) ||
      !vector_ok(rstd) || !vector_ok(dweight) || !vector_ok(dbias))
    return kInvalid;
  if (rows > 0 && cols > 0 && (!mean || !rstd)) return kInvalid;
  if (rows > kMaxDim || cols > kMaxDim) return SGEMM_CUBE_ERR_NOT_SUPPORTED;
  const size_t need = rows && cols ? norm_grad_ws(rows, cols) : 0;
  if (!workspace_ok(ws, ws_bytes, need)) return kInvalid;
  const uint64_t r4 = 4 * static_cast<uint64_t>(rows), c4 = 4 * static_cast<uint64_t>(cols);
  const Span dy{dY, span_bytes(rows, cols, lddy, elem)}, x{X, span_bytes(rows, cols, ldx, elem)};
  const Span dx{dX, span_bytes(rows, cols, lddx, elem)}, w{weight, c4}, mu{mean, r4}, rs{rstd, r4};
  const Span dw{dweight, c4}, db{dbias, c4}, wsp{ws, need};
  const bool in_place = dX == dY && lddx == lddy;
  if ((!in_place && hits(dx, {dy})) || hits(dx, {x, w, mu, rs, dw, db, wsp}) ||
      hits(dw, {dy, x, w, mu, rs, db, wsp}) || hits(db, {dy, x, w, mu, rs, wsp}) ||
      hits(wsp, {dy, x, w, mu, rs}))
    return kInvalid;
  if (cols == 0) return SGEMM_CUBE_OK;
  const NormGradArgs a{rows, cols, dY, lddy, X, ldx, weight, mean, rstd, dX, lddx, dweight, dbias,
                       static_cast<float*>(ws)};
  return status_of(launch_norm_grad(a, dtype, stream));
}

int sgemm_cube_adamw(int64_t tensors, const sgemm_cube_adamw_tensor_t* list, int grad_dtype,
                     int state_bits, double lr, double beta1, double beta2, double eps,
                     double grad_scale, int64_t step, hipStream_t stream) {
  using namespace sgc;
  if (!valid_dtype(grad_dtype) || step < 1) return kInvalid;
  if (!std::isfinite(lr) || !(eps >= 0.0) || std::isinf(eps) || !(beta1 >= 0.0 && beta1 < 1.0) ||
      !(beta2 >= 0.0 && beta2 < 1.0) || !std::isfinite(grad_scale))
    return kInvalid;
  if (const int st = check_adamw_list(tensors, list, state_bits); st != SGEMM_CUBE_OK) return st;
  const uint64_t elem = dtype_bytes(grad_dtype);
  for (int64_t i = 0; i < tensors; ++i) {
    const sgemm_cube_adamw_tensor_t& t = list[i];
    if (t.count == 0) continue;
    if (!t.param || !vector_ok(t.param) || !t.grad ||
        reinterpret_cast<uintptr_t>(t.grad) % elem != 0 || !std::isfinite(t.weight_decay))
      return kInvalid;
    const uint64_t n = static_cast<uint64_t>(t.count), blocks = (n + kAdamwBlock - 1) / kAdamwBlock;
    const uint64_t state = n * (state_bits / 8), scale = state_bits == 8 ? 4 * blocks : 0;
    const Span p{t.param, 4 * n}, g{t.grad, elem * n}, m{t.exp_avg, state}, v{t.exp_avg_sq, state};
    const Span ms{t.exp_avg_scale, scale}, vs{t.exp_avg_sq_scale, scale};
    if (hits(p, {g, m, v, ms, vs}) || hits(m, {g, v, ms, vs}) || hits(v, {g, ms, vs}) ||
        hits(ms, {g, vs}) || hits(vs, {g}))
      return kInvalid;
  }
  AdamwHyper h;
  h.beta1 = static_cast<float>(beta1);
  h.rest1 = static_cast<float>(1.0 - beta1);
  h.beta2 = static_cast<float>(beta2);
  h.rest2 = static_cast<float>(1.0 - beta2);
  h.eps = static_cast<float>(eps);
  h.grad_scale = static_cast<float>(grad_scale);
  h.step_size = static_cast<float>(lr / (1.0 - std::pow(beta1, static_cast<double>(step))));
  h.root = static_cast<float>(1.0 / std::sqrt(1.0 - std::pow(beta2, static_cast<double>(step))));
  return status_of(launch_adamw(tensors, list, grad_dtype, state_bits, lr, h, stream));
}

int sgemm_cube_adamw_values(int64_t tensors, const sgemm_cube_adamw_tensor_t* list,
                            float* const* exp_avg, float* const* exp_avg_sq,
                            hipStream_t stream) {
  using namespace sgc;
  if (const int st = check_adamw_list(tensors, list, 8); st != SGEMM_CUBE_OK) return st;
  if (tensors > 0 && (!exp_avg || !exp_avg_sq)) return kInvalid;
  for (int64_t i = 0; i < tensors; ++i) {
    const sgemm_cube_adamw_tensor_t& t = list[i];
    if (t.count == 0) continue;
    if (!exp_avg[i] || !vector_ok(exp_avg[i]) || !exp_avg_sq[i] || !vector_ok(exp_avg_sq[i]))
      return kInvalid;
    const uint64_t n = static_cast<uint64_t>(t.count), blocks = (n + kAdamwBlock - 1) / kAdamwBlock;
    const Span m{t.exp_avg, n}, v{t.exp_avg_sq, n}, ms{t.exp_avg_scale, 4 * blocks};
    const Span vs{t.exp_avg_sq_scale, 4 * blocks};
    const Span mo{exp_avg[i], 4 * n}, vo{exp_avg_sq[i], 4 * n};
    if (hits(mo, {m, v, ms, vs, vo}) || hits(vo, {m, v, ms, vs})) return kInvalid;
  }
  return status_of(launch_adamw_values(tensors, list, exp_avg, exp_avg_sq, stream));
}

}  // extern "C"
#pragma GCC visibility pop
