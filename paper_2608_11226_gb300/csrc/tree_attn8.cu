// Attention of new tokens (tree_attn.cuh) over 8-bit caches.
#include "tree_attn.cuh"

namespace pe {

static __device__ int32_t g_gave_up8 = 0;

pe_status read_flag(const void* symbol, bool* set);

pe_status tree_attn8_check(bool* gave_up) { return read_flag(&g_gave_up8, gave_up); }

pe_status tree_attn8_launch(const TreeArgs& a, void* ws, const Patience& patience, cudaStream_t st) {
  int32_t* error;
  const pe_status s = tree::flag_address(&g_gave_up8, &error);
  if (s != PE_OK) return s;
  return a.dtype == PE_BF16 ? tree::go_dim<__nv_bfloat16, true>(a, ws, error, patience, st) : tree::go_dim<__half, true>(a, ws, error, patience, st);
}

}  // namespace pe
