// Attention of new tokens (tree_attn.cuh) over 8-bit caches.
#include "tree_attn.cuh"

namespace pe {

pe_status tree_attn8_launch(const TreeArgs& a, void* ws, int32_t* error, const Patience& patience, cudaStream_t st) {
  return a.dtype == PE_BF16 ? tree::go_dim<__nv_bfloat16, true>(a, ws, error, patience, st) : tree::go_dim<__half, true>(a, ws, error, patience, st);
}

}  // namespace pe
