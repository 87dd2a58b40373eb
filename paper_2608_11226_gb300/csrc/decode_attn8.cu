// One-token attention (decode_attn.cuh) over 8-bit caches.
#include "decode_attn.cuh"

namespace pe {

int64_t decode_attn8_ws_bytes(const pe_kv_cache& c, int n_q_heads) { return decode_ws_bytes(c, n_q_heads); }

template <typename T, int D>
static pe_status go_heads(const DecodeArgs& a, void* ws, cudaStream_t st) {
  const int n = seg_heads(D, a.n_q_heads / a.c.n_heads);
  if (n == 8) return go<T, true, D, 1, 1>(a, ws, st);
  if (n == 16) return go<T, true, D, D == 256 ? 1 : 2, D == 256 ? 2 : 1>(a, ws, st);
  if constexpr (D == 64)
    if (n == 32) return go<T, true, D, 4, 1>(a, ws, st);
  if constexpr (D < 256)
    if (n == 24) return go<T, true, D, 3, 1>(a, ws, st);
  return fail(PE_EINVAL, "too many heads");  // they go to tree_attn_launch
}

template <typename T>
static pe_status go_dim(const DecodeArgs& a, void* ws, cudaStream_t st) {
  if (a.c.head_dim == 64) return go_heads<T, 64>(a, ws, st);
  if (a.c.head_dim == 128) return go_heads<T, 128>(a, ws, st);
  return go_heads<T, 256>(a, ws, st);
}

pe_status decode_attn8_launch(const DecodeArgs& a, int dtype, void* ws, cudaStream_t st) {
  ProfScope ps(PE_PROF_DECODE_ATTN, st);
  return dtype == PE_BF16 ? go_dim<__nv_bfloat16>(a, ws, st) : go_dim<__half>(a, ws, st);
}

}  // namespace pe
