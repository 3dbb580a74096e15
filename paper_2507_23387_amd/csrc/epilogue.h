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
template <class Epi>
constexpr bool kThroughLds = std::is_same<Epi, Epilogue>::value;

// The shifts of a wave's kBlocks x 16 rows (or columns) from `first` on, 64 lines at a
// time, one a lane, which hand them out: all of a lane's own are more than the wide
// kernels' accumulators leave registers for.  Lines past the end take the last one's;
// they are not stored.
template <int kBlocks>
struct LineShifts {
  int held[(kBlocks + 3) / 4];
  __device__ __forceinline__ LineShifts(const int* shift, int first, int lines) {
#pragma unroll
    for (int h = 0; h < (kBlocks + 3) / 4; ++h)
      held[h] = shift[min(first + 64 * h + static_cast<int>(threadIdx.x & 63), lines - 1)];
  }
  // That of line i of block b.
  __device__ __forceinline__ int of(int b, int i) const {
    return __shfl(held[b / 4], b % 4 * 16 + i);
  }
};

// store_tile16, for Unscale each entry times 2^-shift of its row or column.
template <int kSubM, int kSubN, class Epi, typename F>
__device__ __forceinline__ void store_product(const Epi& epi, float* __restrict__ C, int64_t ldc,
                                              int M, int N, int row0, int col0, bool full,
                                              F value) {
  if constexpr (!std::is_same<Epi, Unscale>::value) {
    store_tile16<kSubM, kSubN>(C, ldc, M, N, row0, col0, full, value);
  } else if (epi.columns) {
    const int i0 = threadIdx.x & 15;
    const LineShifts<kSubN> lines(epi.shift, col0 - i0, N);
    int q[kSubN];
#pragma unroll
    for (int j = 0; j < kSubN; ++j) q[j] = -lines.of(j, i0);
    store_tile16<kSubM, kSubN>(C, ldc, M, N, row0, col0, full, [&](int i, int j, int r) {
      return __builtin_ldexpf(value(i, j, r), q[j]);
    });
  } else {
    const int i0 = 4 * ((threadIdx.x & 63) >> 4);
    const LineShifts<kSubM> lines(epi.shift, row0 - i0, M);
    float* const base = C + static_cast<int64_t>(row0) * ldc + col0;
#pragma unroll
    for (int i = 0; i < kSubM; ++i) {
      int p[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) p[r] = -lines.of(i, i0 + r);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int rr = i * 16 + r;
        float* const at = base + static_cast<int64_t>(rr) * ldc;
#pragma unroll
        for (int j = 0; j < kSubN; ++j)
          if (full || (row0 + rr < M && col0 + j * 16 < N))
            at[j * 16] = __builtin_ldexpf(value(i, j, r), p[r]);
      }
      SCHED_FENCE();
    }
  }
}

// Keeps the tile's indices in scalar registers.  The epilogue uses them lane by
// lane too, and where the compiler therefore holds them in vector registers it
// moves the copies' base addresses to scalar ones right before each dma16s, whose
// inline asm it gives none of the 5 wait states that a VMEM instruction needs
// after a vector instruction wrote its scalar base (tests/test_asm_hazards.py).
template <class Epi>
__device__ __forceinline__ void scalar_tile(int& tm, int& tn) {
  if constexpr (!std::is_same<Epi, NoEpilogue>::value) {
    tm = __builtin_amdgcn_readfirstlane(tm);
    tn = __builtin_amdgcn_readfirstlane(tn);
  }
}

// Four adjacent floats at any address that floats have.
typedef float floatx4_any __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ floatx4 load_any(const float* p) {
  return *reinterpret_cast<const floatx4_any*>(p);
}
__device__ __forceinline__ void store_any(float* p, floatx4 v) {
  *reinterpret_cast<floatx4_any*>(p) = v;
}

// Accumulator blocks (16 rows) that a wave of kWaves stages at a time in
// `bytes` of LDS, at kCols columns of 16.
constexpr int epilogue_chunk(int rows, int cols, int waves, size_t bytes) {
  int c = rows;
  while (c > 1 && static_cast<size_t>(waves) * c * cols * 1024 > bytes) --c;
  return c;
}

// One piece of a row at the end of the matrix: entry (gr, gc) and up to three
// beside it.
__device__ __forceinline__ void epilogue_edge(const Epilogue& e, float* Y, int64_t ldy, int M,
                                              int N, int gr, int gc, floatx4 v) {
  if (gr >= M) return;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (gc + k >= N) break;
    float x = v[k];
    if (e.bias) x += e.bias[gc + k];
    if (e.z) e.z[static_cast<int64_t>(gr) * e.ldz + gc + k] = x;
    x = activate(e.activation, x);
    if (e.r) x += e.r[static_cast<int64_t>(gr) * e.ldr + gc + k];
    Y[static_cast<int64_t>(gr) * ldy + gc + k] = x;
  }
}

// Y = act(Z) + R, Z = value(i, j, r) + bias for a wave's kSubM x kSubN accumulators
// of 16 x 16 (store_tile16's layout; row0, col0: its first row and column).  kChunk
// rows of blocks at a time go through `stage`, the wave's own LDS, so that lane l
// then has four adjacent columns: bias, residual, Z and Y move in 16-byte pieces of
// whole rows, and the activation is one rolled loop of four pieces and not one copy
// per accumulator (one piece at a time, a lone wave per SIMD waited out each step of
// it: 8192 x 8192 x 4096 with GELU and Z 1289 us in all, so 1199 to 1269, of which
// the split is 94 to 98; the product alone 1170 to 1198).  Column c of row r is at
// c ^ 16 ((r / 4) % 4) of the row (as far as its width allows), which spreads the 4
// row groups of an accumulator over the banks.
template <int kSubM, int kSubN, int kChunk, typename F>
__device__ __forceinline__ void epilogue_tile(const Epilogue& e, float* stage, float* Y,
                                              int64_t ldy, int M, int N, int row0, int col0,
                                              F value) {
  constexpr int kWidth = 16 * kSubN, kQuads = kWidth / 4;
  constexpr int kSwap = kSubN % 4 == 0 ? 3 : kSubN % 2 == 0 ? 1 : 0;
  const int lane = threadIdx.x & 63;
  const bool full = row0 + 16 * kSubM <= M && col0 + kWidth <= N;
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
        // Row by row, so that no more accumulators are read ahead than there are
        // registers for.
        SCHED_FENCE();
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    constexpr int kPieces = kN * kSubN;  // of this lane
    constexpr int kU = kPieces % 4 == 0 ? 4 : kPieces % 2 == 0 ? 2 : 1;
#pragma unroll 1
    for (int p0 = 0; p0 < kPieces; p0 += kU) {
      floatx4 v[kU];
      int gr[kU], gc[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int q = lane + 64 * (p0 + u), row = q / kQuads, c = 4 * (q - row * kQuads);
        gr[u] = row0 + 16 * i0 + row;
        gc[u] = col0 + c;
        v[u] = *reinterpret_cast<const floatx4*>(stage + row * kWidth +
                                                 (c ^ (((row >> 2) & kSwap) << 4)));
      }
      if (!full) {
#pragma unroll
        for (int u = 0; u < kU; ++u) epilogue_edge(e, Y, ldy, M, N, gr[u], gc[u], v[u]);
        continue;
      }
      floatx4 r[kU];
      if (e.r) {
#pragma unroll
        for (int u = 0; u < kU; ++u)
          r[u] = load_any(e.r + static_cast<int64_t>(gr[u]) * e.ldr + gc[u]);
      }
      if (e.bias) {
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const floatx4 b = load_any(e.bias + gc[u]);
#pragma unroll
          for (int k = 0; k < 4; ++k) v[u][k] += b[k];
        }
      }
      if (e.z) {
#pragma unroll
        for (int u = 0; u < kU; ++u)
          store_any(e.z + static_cast<int64_t>(gr[u]) * e.ldz + gc[u], v[u]);
      }
      activate_all(e.activation, v);
      if (e.r) {
#pragma unroll
        for (int u = 0; u < kU; ++u)
#pragma unroll
          for (int k = 0; k < 4; ++k) v[u][k] += r[u][k];
      }
#pragma unroll
      for (int u = 0; u < kU; ++u)
        store_any(Y + static_cast<int64_t>(gr[u]) * ldy + gc[u], v[u]);
    }
  });
}

}  // namespace
}  // namespace sgc
