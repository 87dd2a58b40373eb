// Attention of new tokens (tree_attn.cuh): workspace, dispatch, 16-bit caches.
#include "tree_attn.cuh"

namespace pe {

pe_status tree_attn8_launch(const TreeArgs& a, void* ws, int32_t* error, const Patience& patience, cudaStream_t st);
pe_status tc_error_flag(int32_t** p);        // mlp_bf16.cu
pe_status device_check(cudaStream_t st);

int64_t tree_attn_ws_bytes(const pe_kv_cache& c, int n_nodes, int n_q_heads) {
  const int rows = tree::wide(c.head_dim, n_nodes * (n_q_heads / c.n_heads)) ? 256 : 128;
  return tree::kMetaBytes + 2 * (int64_t)tree::kCtas * rows * (c.head_dim + 2) * 4;  // two pieces for each CTA
}

pe_status tree_attn_launch(const TreeArgs& a, void* ws, cudaStream_t st, const Patience& patience) {
  ProfScope ps(a.mask ? PE_PROF_TREE_ATTN : PE_PROF_DECODE_ATTN, st);
  int32_t* error;  // set when a wait gives up
  const pe_status s = tc_error_flag(&error);
  if (s != PE_OK) return s;
  if (a.c.dtype == PE_E4M3) return tree_attn8_launch(a, ws, error, patience, st);
  return a.dtype == PE_BF16 ? tree::go_dim<__nv_bfloat16, false>(a, ws, error, patience, st) : tree::go_dim<__half, false>(a, ws, error, patience, st);
}

// Self-test of the waits: a narrow and a wide block of rows whose tiles are never placed.  ws: 2^26 bytes, in
// which a cache of four pages, a table, queries and the workspace of the call find room.
pe_status tree_attn_selftest(bool eight, long long limit, void* ws, cudaStream_t st) {
  constexpr int kPages = 4, kPage = 64, kDim = 128, kSeqs = 2, kNodes = 64, kHeads = 3;
  char* at = reinterpret_cast<char*>(ws);
  auto take = [&](int64_t bytes) {
    char* p = at;
    at += (bytes + 255) / 256 * 256;
    return p;
  };
  const int64_t cells = kPages * kPage;
  TreeArgs a{};
  a.c = pe_kv_cache{};
  a.c.k = take(cells * kDim * 2), a.c.v = take(cells * kDim * 2);
  a.sc.k = reinterpret_cast<uint8_t*>(take(cells)), a.sc.v = reinterpret_cast<uint8_t*>(take(cells));
  a.sc.page_stride = kPage, a.sc.slot_stride = 1;
  a.c.table = reinterpret_cast<int32_t*>(take(kSeqs * kPages * 4));
  a.q = take((int64_t)kSeqs * kNodes * kHeads * kDim * 2), a.out = take((int64_t)kSeqs * kNodes * kHeads * kDim * 2);
  char* zeros = at;
  a.lens = reinterpret_cast<int32_t*>(take(kSeqs * 4));
  a.mask = reinterpret_cast<uint64_t*>(take(kSeqs * kNodes * 8));
  PE_TRY_CUDA(cudaMemsetAsync(ws, 0, zeros - reinterpret_cast<char*>(ws), st));
  PE_TRY_CUDA(cudaMemsetAsync(zeros, 1, at - zeros, st));  // every length beyond the table; node 0 of every eight
  a.c.n_pages = kPages, a.c.page_stride = kPage * kDim, a.c.slot_stride = kDim, a.c.table_stride = kPages;
  a.c.n_seqs = kSeqs, a.c.max_pages = kPages, a.c.page_size = kPage, a.c.n_heads = 1, a.c.head_dim = kDim;
  a.c.dtype = eight ? PE_E4M3 : PE_BF16;
  a.q_seq = a.o_seq = kNodes * kHeads * kDim, a.q_node = a.o_node = kHeads * kDim, a.q_head = a.o_head = kDim;
  a.scale = 1.0f, a.n_nodes = kNodes, a.dtype = PE_BF16, a.mask_stride = kNodes;
  bool gave_up = false;
  for (int heads : {1, kHeads}) {
    a.n_q_heads = heads;
    if (at - reinterpret_cast<char*>(ws) + tree_attn_ws_bytes(a.c, kNodes, heads) > (int64_t)1 << 26) return fail(PE_ESTATE, "self-test needs more room");
    Patience p;
    p.clocks = limit, p.hold = true;
    const pe_status s = tree_attn_launch(a, at, st, p);
    if (s != PE_OK) return s;
    const pe_status r = device_check(st);
    if (r != PE_OK && r != PE_ETIMEOUT) return r;
    gave_up |= r == PE_ETIMEOUT;
  }
  return gave_up ? fail(PE_ETIMEOUT, "bounded waits of the attention kernel gave up (self-test)") : PE_OK;
}

}  // namespace pe
