// Argument checks shared by the C-ABI layers of libsgemmcube (api.hip,
// layers_api.hip).  Internal.
#pragma once

#include <cmath>
#include <cstdint>

#include "internal.h"
#include "sgemm_cube.h"

namespace sgc {

// Largest dimension the kernels index with 32-bit tile arithmetic; also keeps
// every grid dimension within its hardware limit.
constexpr int64_t kMaxDim = (int64_t{1} << 30);

inline bool valid_order(int order) {
  return order == SGEMM_CUBE_ELEMENTWISE || order == SGEMM_CUBE_TERMWISE ||
         order == SGEMM_CUBE_ELEMENTWISE_CROSS_FIRST;
}

// Public accumulation order -> internal kernel variant.
inline int variant_of(int order) {
  switch (order) {
    case SGEMM_CUBE_ELEMENTWISE: return kElementwise;
    case SGEMM_CUBE_TERMWISE: return kTermwise;
    default: return kCrossFirst;
  }
}

inline bool valid_scale(float s) {
  if (!std::isfinite(s) || s < 1.0f || s > 16777216.0f) return false;
  int e = 0;
  return std::frexp(s, &e) == 0.5f;  // exact power of two
}

// Bytes spanned by a rows x cols row-major matrix with leading dimension ld.
inline uint64_t span_bytes(int64_t rows, int64_t cols, int64_t ld, uint64_t elem) {
  if (rows <= 0 || cols <= 0) return 0;
  return (static_cast<uint64_t>(rows - 1) * static_cast<uint64_t>(ld) +
          static_cast<uint64_t>(cols)) * elem;
}

inline bool overlap(const void* p, uint64_t pn, const void* q, uint64_t qn) {
  if (pn == 0 || qn == 0) return false;
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return a < b + qn && b < a + pn;
}

// Grid limits: GEMM workgroups (at most (Mp / 256) * (Np / 128) of the wide
// kernels) must fit an int, and B has at most 65535 panels (Np / 128).
inline bool round_up_tiles_exceed(int64_t M, int64_t N) {
  const int64_t Mp = round_up(M, kRowPad), Np = round_up(N, kRowPad);
  return (Mp / 256) * (Np / 128) > INT32_MAX || Np / kPanel > 65535;
}

// ld * rows must not overflow int64 when forming addresses.
inline bool ld_ok(int64_t rows, int64_t ld) {
  return rows <= 1 || ld <= INT64_MAX / 8 / rows;
}

}  // namespace sgc
