// Attention of one new token per sequence over a paged cache (formulas:
// pe.h).  One CTA per (sequence, query head); a warp takes every fourth
// position with a running maximum and sum, the warps join at the end.
#include <math_constants.h>

#include "tokens.cuh"

namespace pe {

template <typename T, int D>
__global__ void __launch_bounds__(128) decode_attn_kernel(DecodeArgs a) {
  constexpr int E = D / 32;
  __shared__ float sm[4], sl[4], so[4][D];
  const int h = blockIdx.x, b = blockIdx.y, w = threadIdx.x / 32, lane = threadIdx.x % 32;
  const pe_kv_cache& c = a.c;
  const int hk = h / (a.n_q_heads / c.n_heads);
  const int n = (int)min((int64_t)max(a.lens[b], 0), (int64_t)c.max_pages * c.page_size);
  const int first = a.window > 0 ? max(0, n - a.window) : 0;
  const T* q = (const T*)a.q + b * a.q_seq + h * a.q_head + lane * E;
  float qr[E], o[E], m = -CUDART_INF_F, l = 0.0f;
  for (int i = 0; i < E; ++i) {
    qr[i] = to_f32(q[i]);
    o[i] = 0.0f;
  }
  for (int j = first + w; j < n; j += 4) {
    const int page = c.table[(int64_t)b * c.table_stride + j / c.page_size];
    if (page < 0 || page >= c.n_pages) continue;
    const int64_t at = kv_page_offset(c, page) + (int64_t)(j % c.page_size) * c.slot_stride + hk * c.head_stride + lane * E;
    const T* k = (const T*)c.k + at;
    const T* v = (const T*)c.v + at;
    float s = 0.0f;
    for (int i = 0; i < E; ++i) s = fmaf(qr[i], to_f32(k[i]), s);
    for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    s *= a.scale;
    if (s == -CUDART_INF_F) continue;
    const float mn = fmaxf(m, s);
    const float f = expf(m - mn), p = expf(s - mn);
    m = mn;
    l = l * f + p;
    for (int i = 0; i < E; ++i) o[i] = o[i] * f + p * to_f32(v[i]);
  }
  for (int i = 0; i < E; ++i) so[w][lane * E + i] = o[i];
  if (lane == 0) {
    sm[w] = m;
    sl[w] = l;
  }
  __syncthreads();
  if (w) return;
  const float mm = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
  float f[4], L = 0.0f;
  for (int x = 0; x < 4; ++x) {
    f[x] = sm[x] == -CUDART_INF_F ? 0.0f : expf(sm[x] - mm);
    L += f[x] == 0.0f ? 0.0f : f[x] * sl[x];
  }
  T* out = (T*)a.out + b * a.o_seq + h * a.o_head + lane * E;
  for (int i = 0; i < E; ++i) {
    float r = 0.0f;
    for (int x = 0; x < 4; ++x)
      if (f[x] != 0.0f) r += f[x] * so[x][lane * E + i];
    out[i] = from_f32<T>(L == 0.0f ? 0.0f : r / L);
  }
  if (lane == 0 && a.lse) a.lse[(int64_t)b * a.n_q_heads + h] = L == 0.0f ? -CUDART_INF_F : mm + logf(L);
}

int64_t decode_attn_ws_bytes(const pe_kv_cache&, int) { return 0; }

template <typename T>
static void go(const DecodeArgs& a, cudaStream_t st) {
  const dim3 grid(a.n_q_heads, a.c.n_seqs);
  if (a.c.head_dim == 64)
    decode_attn_kernel<T, 64><<<grid, 128, 0, st>>>(a);
  else if (a.c.head_dim == 128)
    decode_attn_kernel<T, 128><<<grid, 128, 0, st>>>(a);
  else
    decode_attn_kernel<T, 256><<<grid, 128, 0, st>>>(a);
}

pe_status decode_attn_launch(const DecodeArgs& a, void*, cudaStream_t st) {
  ProfScope ps(PE_PROF_DECODE_ATTN, st);
  if (a.c.n_seqs > 65535) return fail(PE_EINVAL, "n_seqs too large");
  if (a.c.dtype == PE_BF16)
    go<__nv_bfloat16>(a, st);
  else
    go<__half>(a, st);
  PE_CHECK_LAUNCH("decode_attn");
  return PE_OK;
}

}  // namespace pe
