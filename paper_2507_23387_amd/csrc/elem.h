// Elements of the layers' three types, in pieces of 16 bytes.  Internal; every
// function has internal linkage.
#pragma once

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

// The same piece as it lies.
template <int kDtype>
__device__ __forceinline__ typename Elem<kDtype>::Piece raw_piece(
    const typename Elem<kDtype>::T* row, int j, int n) {
  using L = Elem<kDtype>;
  typename L::Piece p;
  if (j + L::kE <= n) {
    p = *reinterpret_cast<const typename L::Piece*>(row + j);
  } else {
#pragma unroll
    for (int e = 0; e < L::kE; ++e)
      p[e] = j + e < n ? row[j + e] : static_cast<typename L::T>(0.0f);
  }
  return p;
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

}  // namespace
}  // namespace sgc
