// Attention of new tokens (tree_attn.cuh): workspace, dispatch, 16-bit caches.
#include "tree_attn.cuh"

namespace pe {

static __device__ int32_t g_gave_up = 0;

pe_status tree_attn8_launch(const TreeArgs& a, void* ws, cudaStream_t st);
pe_status tree_attn8_check(bool* gave_up);

// reads and clears a flag; the caller has waited for the launches
pe_status read_flag(const void* symbol, bool* set) {
  int32_t v = 0;
  PE_TRY_CUDA(cudaMemcpyFromSymbol(&v, symbol, sizeof(v)));
  if (v) {
    *set = true;
    v = 0;
    PE_TRY_CUDA(cudaMemcpyToSymbol(symbol, &v, sizeof(v)));
  }
  return PE_OK;
}

pe_status tree_attn_check(bool* gave_up) {
  const pe_status s = read_flag(&g_gave_up, gave_up);
  return s != PE_OK ? s : tree_attn8_check(gave_up);
}

int64_t tree_attn_ws_bytes(const pe_kv_cache& c, int n_nodes, int n_q_heads) {
  const int rows = tree::wide(c.head_dim, n_nodes * (n_q_heads / c.n_heads)) ? 256 : 128;
  return tree::kMetaBytes + 2 * (int64_t)tree::kCtas * rows * (c.head_dim + 2) * 4;  // two pieces for each CTA
}

pe_status tree_attn_launch(const TreeArgs& a, void* ws, cudaStream_t st) {
  ProfScope ps(a.mask ? PE_PROF_TREE_ATTN : PE_PROF_DECODE_ATTN, st);
  if (a.c.dtype == PE_E4M3) return tree_attn8_launch(a, ws, st);
  int32_t* error;
  const pe_status s = tree::flag_address(&g_gave_up, &error);
  if (s != PE_OK) return s;
  return a.dtype == PE_BF16 ? tree::go_dim<__nv_bfloat16, false>(a, ws, error, st) : tree::go_dim<__half, false>(a, ws, error, st);
}

}  // namespace pe
