// C entry points of the token operators: argument checks, all before any
// launch, and dispatch.
#include <cmath>

#include "tokens.cuh"

using namespace pe;

static bool off(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// a stride of vectors that are read 16 bytes at a time
static bool bad_stride(int64_t s) { return s < 0 || (s & 7) != 0 || s > ((int64_t)1 << 44); }

static bool is16(int32_t dtype) { return dtype == PE_BF16 || dtype == PE_F16; }

// `eight`: a cache of 8-bit codes will do
static pe_status check_cache(const pe_kv_cache* c, bool eight = false) {
  if (!c) return fail(PE_EINVAL, "null cache");
  if (!is16(c->dtype) && !(eight && c->dtype == PE_E4M3))
    return fail(PE_EINVAL, eight ? "cache dtype must be PE_BF16, PE_F16 or PE_E4M3" : "cache dtype must be PE_BF16 or PE_F16");
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return fail(PE_EINVAL, "head_dim must be 64, 128 or 256");
  if (c->n_heads < 1 || c->n_heads > 1024) return fail(PE_EINVAL, "n_heads must be in [1, 1024]");
  if (c->page_size < 1 || c->page_size > 65536) return fail(PE_EINVAL, "page_size must be in [1, 65536]");
  if (c->n_pages < 1 || c->n_pages > INT32_MAX) return fail(PE_EINVAL, "n_pages must be in [1, 2^31)");
  if (c->n_seqs < 0 || c->n_seqs > (1 << 20)) return fail(PE_EINVAL, "n_seqs must be in [0, 2^20]");
  if (c->max_pages < 1 || (int64_t)c->max_pages * c->page_size > (1 << 30))
    return fail(PE_EINVAL, "max_pages >= 1 and max_pages * page_size <= 2^30 required");
  if (c->table_stride < 0 || (c->n_seqs > 1 && c->table_stride < c->max_pages))
    return fail(PE_EINVAL, "table_stride must be at least max_pages");
  if (bad_stride(c->page_stride) || bad_stride(c->slot_stride) || bad_stride(c->head_stride))
    return fail(PE_EINVAL, "cache strides must be multiples of 8 elements");
  if (c->dtype == PE_E4M3 && ((c->page_stride | c->slot_stride | c->head_stride) & 15) != 0)
    return fail(PE_EINVAL, "strides of an 8-bit cache must be multiples of 16");
  if (!c->k || !c->v || (!c->table && c->n_seqs > 0)) return fail(PE_EINVAL, "null argument");
  if (off(c->k, 16) || off(c->v, 16)) return fail(PE_EINVAL, "k and v must be 16-byte aligned");
  return PE_OK;
}

static pe_status check_scales(const pe_kv_cache* c, const pe_kv_scales* sc) {
  if (c->dtype != PE_E4M3) return sc ? fail(PE_EINVAL, "a 16-bit cache has no scales") : PE_OK;
  if (!sc || !sc->k || !sc->v) return fail(PE_EINVAL, "an 8-bit cache needs scales");
  const int64_t most = (int64_t)1 << 44;
  if (sc->page_stride < 0 || sc->slot_stride < 0 || sc->head_stride < 0 || sc->page_stride > most || sc->slot_stride > most ||
      sc->head_stride > most)
    return fail(PE_EINVAL, "scale strides must be in [0, 2^44]");
  return PE_OK;
}

// an 8-bit cache with its scales, and the type of what goes in or comes out
static pe_status check_pair(const pe_kv_cache* c, const pe_kv_scales* sc, int32_t dtype) {
  const pe_status s = check_cache(c, true);
  if (s != PE_OK) return s;
  if (!is16(dtype) || (c->dtype != PE_E4M3 && dtype != c->dtype))
    return fail(PE_EINVAL, "dtype must be PE_BF16 or PE_F16, and a 16-bit cache's own");
  return check_scales(c, sc);
}

static pe_status append(const pe_kv_cache* cache, const pe_kv_scales* scales, const pe_kv_tokens* t, const int32_t* slots,
                        int32_t dtype, void* stream) {
  if (!t) return fail(PE_EINVAL, "null tokens");
  if (t->n_tokens < 0 || t->n_tokens > INT32_MAX) return fail(PE_EINVAL, "n_tokens must be in [0, 2^31)");
  if (t->rot_dim < 0 || t->rot_dim > cache->head_dim || t->rot_dim % 16 != 0)
    return fail(PE_EINVAL, "rot_dim must be a multiple of 16 in [0, head_dim]");
  if (t->rot_dim > 0 && (t->max_pos < 1 || t->max_pos > INT32_MAX)) return fail(PE_EINVAL, "max_pos must be in [1, 2^31)");
  if (t->q && (t->n_q_heads < 1 || t->n_q_heads > 65536)) return fail(PE_EINVAL, "n_q_heads must be in [1, 65536]");
  if (t->n_tokens == 0) return PE_OK;
  if (!t->pos || !t->k || !t->v || (t->rot_dim > 0 && !t->rot) || (t->q && !t->q_out)) return fail(PE_EINVAL, "null argument");
  if (bad_stride(t->k_token_stride) || bad_stride(t->k_head_stride) || bad_stride(t->v_token_stride) ||
      bad_stride(t->v_head_stride) ||
      (t->q && (bad_stride(t->q_token_stride) || bad_stride(t->q_head_stride) || bad_stride(t->q_out_token_stride) ||
                bad_stride(t->q_out_head_stride))))
    return fail(PE_EINVAL, "token strides must be multiples of 8 elements");
  if (off(t->k, 16) || off(t->v, 16) || (t->q && (off(t->q, 16) || off(t->q_out, 16))) || (t->rot_dim > 0 && off(t->rot, 16)))
    return fail(PE_EINVAL, "q, q_out, k, v and rot must be 16-byte aligned");
  return kv_append_launch(*cache, scales ? *scales : pe_kv_scales{}, *t, slots, dtype, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" {

pe_status pe_kv_append(const pe_kv_cache* cache, const pe_kv_tokens* t, void* stream) {
  clear_error();
  const pe_status s = check_cache(cache);
  return s != PE_OK ? s : append(cache, nullptr, t, nullptr, cache->dtype, stream);
}

pe_status pe_kv_append_at(const pe_kv_cache* cache, const pe_kv_scales* scales, const pe_kv_tokens* t, const int32_t* slots,
                          int32_t dtype, void* stream) {
  clear_error();
  const pe_status s = check_pair(cache, scales, dtype);
  return s != PE_OK ? s : append(cache, scales, t, slots, dtype, stream);
}

pe_status pe_kv_move(const pe_kv_cache* cache, const pe_kv_scales* scales, const int32_t* src, int64_t src_stride,
                     const int32_t* dst, int64_t dst_stride, int32_t n_moves, void* stream) {
  clear_error();
  pe_status s = check_cache(cache, true);
  if (s == PE_OK) s = check_scales(cache, scales);
  if (s != PE_OK) return s;
  if (n_moves < 0 || n_moves > 64) return fail(PE_EINVAL, "n_moves must be in [0, 64]");
  if (cache->n_seqs > 1 && (src_stride < n_moves || dst_stride < n_moves)) return fail(PE_EINVAL, "src_stride and dst_stride must be at least n_moves");
  if (src_stride < 0 || dst_stride < 0 || src_stride > ((int64_t)1 << 40) || dst_stride > ((int64_t)1 << 40))
    return fail(PE_EINVAL, "src_stride and dst_stride must be in [0, 2^40]");
  if (cache->n_seqs == 0 || n_moves == 0) return PE_OK;
  if (!src || !dst) return fail(PE_EINVAL, "null argument");
  MoveArgs a{*cache, scales ? *scales : pe_kv_scales{}, src, dst, src_stride, dst_stride, n_moves};
  return kv_move_launch(a, reinterpret_cast<cudaStream_t>(stream));
}

static bool bad_group(const pe_kv_cache* c, int32_t n_q_heads) {
  return n_q_heads < 1 || n_q_heads > 65536 || n_q_heads % c->n_heads != 0;
}

static int64_t tree_ws_bytes(const pe_kv_cache& c, int n_nodes, int n_q_heads) {
  return few_rows(c, n_nodes, n_q_heads) ? few_rows_ws_bytes(c, n_nodes, n_q_heads) : tree_attn_ws_bytes(c, n_nodes, n_q_heads);
}

int64_t pe_tree_attn_workspace_bytes(const pe_kv_cache* cache, int32_t n_nodes, int32_t n_q_heads) {
  if (check_cache(cache, true) != PE_OK) return -1;
  if (bad_group(cache, n_q_heads) || n_nodes < 0 || n_nodes > 64) return -1;
  return n_nodes == 0 ? 0 : tree_ws_bytes(*cache, n_nodes, n_q_heads);
}

static pe_status check_workspace(const void* workspace, int64_t bytes, int64_t need) {
  if (need > 0 && !workspace) return fail(PE_EINVAL, "null argument");
  if (bytes < need) return fail(PE_EINVAL, "workspace too small (%lld < %lld bytes)", (long long)bytes, (long long)need);
  if (need > 0 && off(workspace, 256)) return fail(PE_EINVAL, "workspace must be 256-byte aligned");
  return PE_OK;
}

pe_status pe_tree_attn(const pe_kv_cache* cache, const pe_kv_scales* scales, const pe_tree_queries* t, float scale, int32_t window,
                       void* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  if (!t) return fail(PE_EINVAL, "null tree");
  pe_status s = check_pair(cache, scales, t->dtype);
  if (s != PE_OK) return s;
  if (bad_group(cache, t->n_q_heads)) return fail(PE_EINVAL, "n_q_heads must be a multiple of n_heads in [1, 65536]");
  if (t->n_nodes < 0 || t->n_nodes > 64) return fail(PE_EINVAL, "n_nodes must be in [0, 64]");
  if (!std::isfinite(scale)) return fail(PE_EINVAL, "scale must be finite");
  if (window < 0 || (window > 0 && window < 64)) return fail(PE_EINVAL, "window must be 0 or at least 64");
  if (t->mask_stride < 0 || t->mask_stride > ((int64_t)1 << 40)) return fail(PE_EINVAL, "mask_stride must be in [0, 2^40]");
  if (cache->n_seqs == 0 || t->n_nodes == 0) return PE_OK;
  if (!t->q || !t->out || !t->lens || !t->mask) return fail(PE_EINVAL, "null argument");
  if (bad_stride(t->q_seq_stride) || bad_stride(t->q_node_stride) || bad_stride(t->q_head_stride) || bad_stride(t->out_seq_stride) ||
      bad_stride(t->out_node_stride) || bad_stride(t->out_head_stride))
    return fail(PE_EINVAL, "q and out strides must be multiples of 8 elements");
  if (off(t->q, 16) || off(t->out, 16)) return fail(PE_EINVAL, "q and out must be 16-byte aligned");
  if (off(t->mask, 8)) return fail(PE_EINVAL, "mask must be 8-byte aligned");
  s = check_workspace(workspace, workspace_bytes, tree_ws_bytes(*cache, t->n_nodes, t->n_q_heads));
  if (s != PE_OK) return s;
  TreeArgs a{*cache, scales ? *scales : pe_kv_scales{}, t->q, t->out, t->lse, t->lens, t->mask, t->q_seq_stride, t->q_node_stride,
             t->q_head_stride, t->out_seq_stride, t->out_node_stride, t->out_head_stride, t->mask_stride, scale, t->n_nodes,
             t->n_q_heads, window, t->dtype};
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  return few_rows(*cache, t->n_nodes, t->n_q_heads) ? few_rows_launch(a, workspace, st) : tree_attn_launch(a, workspace, st);
}

// Whether one token's heads of a key head are enough for tiles of 128 rows.  Measured
// over 8 bits, 8 key heads, 8 sequences of 32,640 positions, the one-token kernel
// against tiles: head_dim 128, 16 heads 109 against 227 us, 24 heads 153 against 227,
// 32 heads 281 against 226, 64 heads 400 against 229; head_dim 64, 24 heads 94 against
// 170, 32 heads 114 against 170, 64 heads 236 against 171; head_dim 256, 16 heads 208
// against 378, 24 heads 446 against 377.  (Short sequences are latency: 2 of 512,
// 32 heads of 128, 12.3 against 13.4.)
static bool many_heads(const pe_kv_cache& c, int n_q_heads) { return n_q_heads / c.n_heads > (c.head_dim == 256 ? 16 : c.head_dim == 64 ? 32 : 24); }

static int64_t decode8_ws_bytes(const pe_kv_cache& c, int n_q_heads) {
  return many_heads(c, n_q_heads) ? tree_attn_ws_bytes(c, 1, n_q_heads) : decode_attn8_ws_bytes(c, n_q_heads);
}

int64_t pe_decode_attn8_workspace_bytes(const pe_kv_cache* cache, int32_t n_q_heads) {
  if (check_cache(cache, true) != PE_OK || cache->dtype != PE_E4M3 || bad_group(cache, n_q_heads)) return -1;
  return decode8_ws_bytes(*cache, n_q_heads);
}

pe_status pe_decode_attn8(const pe_kv_cache* cache, const pe_kv_scales* scales, int32_t dtype, const void* q,
                          int64_t q_seq_stride, int64_t q_head_stride, int32_t n_q_heads, const int32_t* lens,
                          float scale, int32_t window, void* out, int64_t out_seq_stride, int64_t out_head_stride,
                          float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  pe_status s = check_pair(cache, scales, dtype);
  if (s != PE_OK) return s;
  if (cache->dtype != PE_E4M3) return fail(PE_EINVAL, "cache dtype must be PE_E4M3");
  if (bad_group(cache, n_q_heads)) return fail(PE_EINVAL, "n_q_heads must be a multiple of n_heads in [1, 65536]");
  if (!std::isfinite(scale)) return fail(PE_EINVAL, "scale must be finite");
  if (window < 0) return fail(PE_EINVAL, "window must be >= 0");
  if (cache->n_seqs == 0) return PE_OK;
  if (!q || !out || !lens) return fail(PE_EINVAL, "null argument");
  if (bad_stride(q_seq_stride) || bad_stride(q_head_stride) || bad_stride(out_seq_stride) || bad_stride(out_head_stride))
    return fail(PE_EINVAL, "q and out strides must be multiples of 8 elements");
  if (off(q, 16) || off(out, 16)) return fail(PE_EINVAL, "q and out must be 16-byte aligned");
  s = check_workspace(workspace, workspace_bytes, decode8_ws_bytes(*cache, n_q_heads));
  if (s != PE_OK) return s;
  if (!many_heads(*cache, n_q_heads)) {
    DecodeArgs a{*cache, *scales, q, out, lse, lens, q_seq_stride, q_head_stride, out_seq_stride, out_head_stride, scale, n_q_heads, window};
    return decode_attn8_launch(a, dtype, workspace, reinterpret_cast<cudaStream_t>(stream));
  }
  TreeArgs a{*cache, *scales, q, out, lse, lens, nullptr, q_seq_stride, 0, q_head_stride, out_seq_stride, 0, out_head_stride, 0,
             scale, 1, n_q_heads, window, dtype};
  return tree_attn_launch(a, workspace, reinterpret_cast<cudaStream_t>(stream));
}

int64_t pe_decode_attn_workspace_bytes(const pe_kv_cache* cache, int32_t n_q_heads) {
  if (check_cache(cache) != PE_OK) return -1;
  if (n_q_heads < 1 || n_q_heads > 65536 || n_q_heads % cache->n_heads != 0) return -1;
  return decode_attn_ws_bytes(*cache, n_q_heads);
}

pe_status pe_decode_attn(const pe_kv_cache* cache, const void* q, int64_t q_seq_stride, int64_t q_head_stride,
                         int32_t n_q_heads, const int32_t* lens, float scale, int32_t window, void* out,
                         int64_t out_seq_stride, int64_t out_head_stride, float* lse, void* workspace,
                         int64_t workspace_bytes, void* stream) {
  clear_error();
  pe_status s = check_cache(cache);
  if (s != PE_OK) return s;
  if (n_q_heads < 1 || n_q_heads > 65536 || n_q_heads % cache->n_heads != 0)
    return fail(PE_EINVAL, "n_q_heads must be a multiple of n_heads in [1, 65536]");
  if (!std::isfinite(scale)) return fail(PE_EINVAL, "scale must be finite");
  if (window < 0) return fail(PE_EINVAL, "window must be >= 0");
  if (cache->n_seqs == 0) return PE_OK;
  const int64_t need = decode_attn_ws_bytes(*cache, n_q_heads);
  if (!q || !out || !lens || (need > 0 && !workspace)) return fail(PE_EINVAL, "null argument");
  if (bad_stride(q_seq_stride) || bad_stride(q_head_stride) || bad_stride(out_seq_stride) || bad_stride(out_head_stride))
    return fail(PE_EINVAL, "q and out strides must be multiples of 8 elements");
  if (off(q, 16) || off(out, 16)) return fail(PE_EINVAL, "q and out must be 16-byte aligned");
  if (workspace_bytes < need)
    return fail(PE_EINVAL, "workspace too small (%lld < %lld bytes)", (long long)workspace_bytes, (long long)need);
  if (need > 0 && off(workspace, 256)) return fail(PE_EINVAL, "workspace must be 256-byte aligned");
  DecodeArgs a{*cache, pe_kv_scales{}, q, out, lse, lens, q_seq_stride, q_head_stride, out_seq_stride, out_head_stride, scale, n_q_heads, window};
  return decode_attn_launch(a, workspace, reinterpret_cast<cudaStream_t>(stream));
}

static int elem_size(int32_t dtype) { return dtype == PE_F32 ? 4 : dtype == PE_BF16 || dtype == PE_F16 ? 2 : 0; }

static pe_status check_rows(const void* logits, int32_t dtype, int64_t n, int32_t V, int64_t row_stride, float scale) {
  const int e = elem_size(dtype);
  if (!e) return fail(PE_EINVAL, "dtype must be PE_F32, PE_BF16 or PE_F16");
  if (n < 0 || n > INT32_MAX) return fail(PE_EINVAL, "n must be in [0, 2^31)");
  if (V < 1 || V > (1 << 30)) return fail(PE_EINVAL, "V must be in [1, 2^30]");
  if ((n > 1 && row_stride < V) || row_stride < 0 || row_stride > ((int64_t)1 << 40))
    return fail(PE_EINVAL, "row_stride must be at least V");
  if (!(scale >= 1e-4f && scale <= 1e4f)) return fail(PE_EINVAL, "scale must be in [1e-4, 1e4]");
  if (n == 0) return PE_OK;
  if (!logits) return fail(PE_EINVAL, "null argument");
  if (off(logits, e)) return fail(PE_EINVAL, "logits must be element-aligned");
  return PE_OK;
}

pe_status pe_token_logp(const void* logits, int32_t dtype, int64_t n, int32_t V, int64_t row_stride,
                        const int32_t* tokens, float scale, float* logp, float* entropy, float* lse, int32_t top_k,
                        float* top_logp, int32_t* top_id, void* stream) {
  clear_error();
  pe_status s = check_rows(logits, dtype, n, V, row_stride, scale);
  if (s != PE_OK) return s;
  if (top_k < 0 || top_k > 32 || top_k > V) return fail(PE_EINVAL, "top_k must be in [0, min(32, V)]");
  if (n == 0) return PE_OK;
  if ((logp && !tokens) || (top_k > 0 && (!top_logp || !top_id))) return fail(PE_EINVAL, "null argument");
  if (!logp && !entropy && !lse && top_k == 0) return fail(PE_EINVAL, "no output asked for");
  LogpArgs a{logits, tokens, logp, entropy, lse, top_logp, top_id, n, row_stride, V, top_k, scale};
  return token_logp_launch(a, dtype, reinterpret_cast<cudaStream_t>(stream));
}

pe_status pe_token_logp_grad(const void* logits, int32_t dtype, int64_t n, int32_t V, int64_t row_stride,
                             const int32_t* tokens, float scale, const float* lse, const float* entropy,
                             const float* g_logp, const float* g_entropy, void* dlogits, int64_t d_row_stride,
                             void* stream) {
  clear_error();
  pe_status s = check_rows(logits, dtype, n, V, row_stride, scale);
  if (s != PE_OK) return s;
  if ((n > 1 && d_row_stride < V) || d_row_stride < 0 || d_row_stride > ((int64_t)1 << 40))
    return fail(PE_EINVAL, "d_row_stride must be at least V");
  if (n == 0) return PE_OK;
  if (!lse || !dlogits || (g_logp && !tokens) || (g_entropy && !entropy)) return fail(PE_EINVAL, "null argument");
  if (!g_logp && !g_entropy) return fail(PE_EINVAL, "g_logp or g_entropy required");
  if (off(dlogits, elem_size(dtype))) return fail(PE_EINVAL, "dlogits must be element-aligned");
  if (dlogits == logits && n > 1 && d_row_stride != row_stride)
    return fail(PE_EINVAL, "in place needs d_row_stride == row_stride");
  LogpGradArgs a{logits, dlogits, tokens, lse, entropy, g_logp, g_entropy, n, row_stride, d_row_stride, V, scale};
  return token_logp_grad_launch(a, dtype, reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
