// The epilogue of a linear layer as a GEMM kernel applies it to its tile.
// Internal; every function has internal linkage.
#pragma once

#include <type_traits>

#include "activation.h"
#include "gemm_common.h"
#include "layers.h"

namespace sgc {
namespace {

// In place of an epilogue: C is stored as the product (store_tile16).
struct NoEpilogue {};

// Keeps the tile's indices in scalar registers.  The epilogue uses them lane by
// lane too, and where the compiler therefore holds them in vector registers it
// moves the copies' base addresses to scalar ones right before each dma16s, whose
// inline asm it gives none of the 5 wait states that a VMEM instruction needs
// after a vector instruction wrote its scalar base (tests/test_sgpr_hazard.py).
template <class Epi>
__device__ __forceinline__ void scalar_tile(int& tm, int& tn) {
  if constexpr (!std::is_same<Epi, NoEpilogue>::value) {
    tm = __builtin_amdgcn_readfirstlane(tm);
    tn = __builtin_amdgcn_readfirstlane(tn);
  }
}

typedef float floatx4_any __attribute__((ext_vector_type(4), aligned(4)));

// Accumulator blocks (16 rows) that a wave of kWaves stages at a time in
// `bytes` of LDS, at kCols columns of 16.
constexpr int epilogue_chunk(int rows, int cols, int waves, size_t bytes) {
  int c = rows;
  while (c > 1 && static_cast<size_t>(waves) * c * cols * 1024 > bytes) --c;
  return c;
}

// Y = act(Z) + R, Z = 2^-shift value(i, j, r) + bias for a wave's kSubM x kSubN
// accumulators of 16 x 16 (store_tile16's layout; row0, col0: its first row and
// column).  kChunk rows of blocks at a time go through `stage`, the wave's own
// LDS, so that lane l then has four adjacent columns: bias, residual, Z and Y move
// in 16-byte pieces of whole rows, and the activation is one rolled loop and not
// one copy per accumulator.  Column c of row r is at c ^ 16 ((r / 4) % 4) of the
// row (as far as its width allows), which spreads the 4 row groups of an
// accumulator over the banks.
template <int kSubM, int kSubN, int kChunk, typename F>
__device__ __forceinline__ void epilogue_tile(const Epilogue& e, float* stage, float* Y,
                                              int64_t ldy, int M, int N, int row0, int col0,
                                              F value) {
  constexpr int kWidth = 16 * kSubN;
  constexpr int kSwap = kSubN % 4 == 0 ? 3 : kSubN % 2 == 0 ? 1 : 0;
  const int lane = threadIdx.x & 63;
  const int shift = e.max_bits ? -prescale_shift(*e.max_bits, e.target) : 0;
  static_for<(kSubM + kChunk - 1) / kChunk>([&](auto Cc) {
    constexpr int i0 = decltype(Cc)::value * kChunk;
    constexpr int kN = i0 + kChunk <= kSubM ? kChunk : kSubM - i0;
    // The wave's reads of the chunk before are done.
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < kN; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * i + 4 * (lane >> 4) + r, swap = ((lane >> 4) & kSwap) << 4;
#pragma unroll
        for (int j = 0; j < kSubN; ++j)
          stage[row * kWidth + ((16 * j + (lane & 15)) ^ swap)] = value(i0 + i, j, r);
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int q = lane; q < kN * 16 * (kWidth / 4); q += 64) {
      const int row = q / (kWidth / 4), c = 4 * (q - row * (kWidth / 4));
      const int gr = row0 + 16 * i0 + row, gc = col0 + c;
      if (gr >= M || gc >= N) continue;
      floatx4 v = *reinterpret_cast<const floatx4*>(
          stage + row * kWidth + (c ^ (((row >> 2) & kSwap) << 4)));
      if (e.max_bits) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = __builtin_ldexpf(v[k], shift);
      }
      float* const y = Y + static_cast<int64_t>(gr) * ldy + gc;
      const float* const res = e.r ? e.r + static_cast<int64_t>(gr) * e.ldr + gc : nullptr;
      float* const z = e.z ? e.z + static_cast<int64_t>(gr) * e.ldz + gc : nullptr;
      if (gc + 4 <= N) {
        floatx4_any b = {0.0f, 0.0f, 0.0f, 0.0f}, rr = b;
        if (e.bias) b = *reinterpret_cast<const floatx4_any*>(e.bias + gc);
        if (res) rr = *reinterpret_cast<const floatx4_any*>(res);
        if (e.bias) {
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] += b[k];
        }
        if (z) *reinterpret_cast<floatx4_any*>(z) = v;
        activate4(e.activation, v);
        if (res) {
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] += rr[k];
        }
        *reinterpret_cast<floatx4_any*>(y) = v;
      } else {
        for (int k = 0; k < N - gc; ++k) {
          float x = k == 0 ? v[0] : k == 1 ? v[1] : v[2];
          if (e.bias) x += e.bias[gc + k];
          if (z) z[k] = x;
          x = activate(e.activation, x);
          if (res) x += res[k];
          y[k] = x;
        }
      }
    }
  });
}

}  // namespace
}  // namespace sgc
