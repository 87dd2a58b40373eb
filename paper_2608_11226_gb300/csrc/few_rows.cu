// Attention of drafted tokens with few rows a key head on the one-token kernel
// (decode_attn.cuh): workspace, dispatch, 16-bit caches.
#include "few_rows.cuh"

namespace pe {

pe_status few_rows8_launch(const DecodeArgs& a, int dtype, void* ws, cudaStream_t st);

// Which kernel takes a tree: this one up to as many rows as one warp holds (over 8 bits
// of head_dim 256 two), the one of tiles (tree_attn.cuh) beyond.  Measured with 8 key heads, 8 sequences of
// 32,640 positions, this against that: 8 bits, head_dim 128, 8 rows 93 against 228
// us, 16 rows 112, 24 rows 180 (64 sequences of 2,048: 60, 78, 128 against 158; 2 of 512: 10.0, 13.0,
// 16.4 against 14.8); head_dim 64, 24 rows 98, 32 rows 123 against 172 (73, 98 against 135; 12.7,
// 14.4 against 13.7); head_dim 256, 8 rows 172 against 378, 16 rows 210.
// 16 bits, head_dim 128, 8 rows 166 against 179, 16 rows 171 (64 sequences of 2,048: 91, 96
// against 112), 24 rows 175 against 181 (111 against 112; 2 of 512: 16.2 against 13.0);
// head_dim 64, 24 rows 98, 32 rows 112 against 149 (69, 85 against 95; 12.2, 13.5 against
// 11.7); head_dim 256, 8 rows 316 against 337.
bool few_rows(const pe_kv_cache& c, int n_nodes, int n_q_heads) {
  const int rows = n_nodes * (n_q_heads / c.n_heads);
  const bool eight = c.dtype == PE_E4M3;
  return rows <= (c.head_dim == 256 ? (eight ? 16 : 8) : c.head_dim == 64 ? 32 : eight ? 24 : 16);
}

int64_t few_rows_ws_bytes(const pe_kv_cache& c, int n_nodes, int n_q_heads) { return decode_ws_bytes(c, n_nodes * n_q_heads); }

pe_status few_rows_launch(const TreeArgs& a, void* ws, cudaStream_t st) {
  ProfScope ps(PE_PROF_TREE_ATTN, st);
  const DecodeArgs d{a.c, a.sc, a.q, a.out, a.lse, a.lens, a.q_seq, a.q_head, a.o_seq, a.o_head, a.scale, a.n_q_heads, a.window,
                     a.n_nodes, a.mask, a.q_node, a.o_node, a.mask_stride};
  if (a.c.dtype == PE_E4M3) return few_rows8_launch(d, a.dtype, ws, st);
  return a.dtype == PE_BF16 ? few_dim<__nv_bfloat16, false>(d, ws, st) : few_dim<__half, false>(d, ws, st);
}

}  // namespace pe
