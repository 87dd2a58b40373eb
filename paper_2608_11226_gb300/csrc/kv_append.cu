// Keys and values of new tokens into a paged cache; queries and keys are
// rotated by their position on the way (formulas: pe.h).  One thread per
// element pair; HBM-bound: each row is read and written once.
#include "tokens.cuh"

namespace pe {

template <typename T>
__global__ void __launch_bounds__(256) kv_append_kernel(pe_kv_cache c, pe_kv_tokens t) {
  const int64_t tok = blockIdx.x;
  const int D = c.head_dim, rot = t.rot_dim, half = rot / 2;
  const int nq = t.q ? t.n_q_heads : 0;
  const int s = t.seq ? t.seq[tok] : (int)tok;
  const int p = t.pos[tok];
  const int64_t cap = (int64_t)c.max_pages * c.page_size;
  const bool live = p >= 0 && p < cap && (rot == 0 || p < t.max_pos) && s >= 0 && s < c.n_seqs;
  int64_t slot = -1;
  if (live) {
    const int page = c.table[(int64_t)s * c.table_stride + p / c.page_size];
    if (page >= 0 && page < c.n_pages) slot = kv_page_offset(c, page) + (int64_t)(p % c.page_size) * c.slot_stride;
  }
  const float* cs = t.rot + (int64_t)(live ? p : 0) * rot;
  const int work = (nq + 2 * c.n_heads) * (D / 2);
  for (int i = threadIdx.x; i < work; i += blockDim.x) {
    const int head = i / (D / 2), j = i % (D / 2);
    const T* src;
    T* dst;
    bool turn = true;
    if (head < nq) {
      src = (const T*)t.q + tok * t.q_token_stride + head * t.q_head_stride;
      dst = (T*)t.q_out + tok * t.q_out_token_stride + head * t.q_out_head_stride;
    } else if (head < nq + c.n_heads) {
      src = (const T*)t.k + tok * t.k_token_stride + (head - nq) * t.k_head_stride;
      dst = slot < 0 ? nullptr : (T*)c.k + slot + (head - nq) * c.head_stride;
    } else {
      const int h = head - nq - c.n_heads;
      src = (const T*)t.v + tok * t.v_token_stride + h * t.v_head_stride;
      dst = slot < 0 ? nullptr : (T*)c.v + slot + h * c.head_stride;
      turn = false;
    }
    if (!dst) continue;
    int e0, e1;  // pair j: rotated ones first, then the copied rest
    if (j < half) {
      e0 = t.interleaved ? 2 * j : j;
      e1 = t.interleaved ? 2 * j + 1 : j + half;
    } else {
      e0 = 2 * j;
      e1 = 2 * j + 1;
      turn = false;
    }
    T a = src[e0], b = src[e1];
    if (head < nq && !live) {
      a = from_f32<T>(0.0f);
      b = a;
    } else if (turn) {
      const float x = to_f32(a), y = to_f32(b), co = cs[j], si = cs[half + j];
      a = from_f32<T>(x * co - y * si);
      b = from_f32<T>(y * co + x * si);
    }
    dst[e0] = a;
    dst[e1] = b;
  }
}

pe_status kv_append_launch(const pe_kv_cache& c, const pe_kv_tokens& t, cudaStream_t st) {
  ProfScope ps(PE_PROF_KV_APPEND, st);
  if (c.dtype == PE_BF16)
    kv_append_kernel<__nv_bfloat16><<<(unsigned)t.n_tokens, 256, 0, st>>>(c, t);
  else
    kv_append_kernel<__half><<<(unsigned)t.n_tokens, 256, 0, st>>>(c, t);
  PE_CHECK_LAUNCH("kv_append");
  return PE_OK;
}

}  // namespace pe
