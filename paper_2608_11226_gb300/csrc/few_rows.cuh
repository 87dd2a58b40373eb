// Dispatch of the one-token kernel for drafted nodes.
#pragma once

#include "decode_attn.cuh"

namespace pe {

template <typename T, bool E8, int D>
static pe_status few_go(const DecodeArgs& a, void* ws, cudaStream_t st) {
  const int n = seg_heads(D, a.n_nodes * (a.n_q_heads / a.c.n_heads));
  if (n == 8) return go<T, E8, D, 1, 1, true>(a, ws, st);
  if constexpr (D == 256) {
    if constexpr (E8)
      if (n == 16) return go<T, E8, D, 1, 2, true>(a, ws, st);
  } else {
    if (n == 16) return go<T, E8, D, 2, 1, true>(a, ws, st);
    if constexpr (E8 || D == 64)
      if (n == 24) return go<T, E8, D, 3, 1, true>(a, ws, st);
    if constexpr (D == 64)
      if (n == 32) return go<T, E8, D, 4, 1, true>(a, ws, st);
  }
  return fail(PE_EINVAL, "too many rows");  // few_rows() is false for them
}

template <typename T, bool E8>
static pe_status few_dim(const DecodeArgs& a, void* ws, cudaStream_t st) {
  if (a.c.head_dim == 64) return few_go<T, E8, 64>(a, ws, st);
  if (a.c.head_dim == 128) return few_go<T, E8, 128>(a, ws, st);
  return few_go<T, E8, 256>(a, ws, st);
}

}  // namespace pe
