// Attention of one or several new tokens over a paged cache of 16 or 8 bits
// (formulas: pe.h).  One warp for each row (node and query head).
#include <math_constants.h>

#include "tokens.cuh"

namespace pe {

constexpr int kRowWarps = 4;

__device__ __forceinline__ float2 e4m3_pair(uint16_t w) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(w));
  return unpack2<__half>(h);
}

// two neighbouring elements of a row
template <typename E> __device__ __forceinline__ float2 load2(const void* base, int64_t at) {
  return unpack2<E>(*reinterpret_cast<const uint32_t*>((const E*)base + at));
}
template <> __device__ __forceinline__ float2 load2<uint8_t>(const void* base, int64_t at) {
  return e4m3_pair(*reinterpret_cast<const uint16_t*>((const uint8_t*)base + at));
}

template <typename T, typename E, int D>
__global__ void __launch_bounds__(32 * kRowWarps) tree_rows_kernel(TreeArgs a) {
  const pe_kv_cache& c = a.c;
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * kRowWarps + threadIdx.x / 32;
  pdl_enter();
  if (row >= (int64_t)c.n_seqs * a.n_nodes * a.n_q_heads) return;
  const int h = (int)(row % a.n_q_heads), node = (int)(row / a.n_q_heads % a.n_nodes), b = (int)(row / a.n_q_heads / a.n_nodes);
  const int hk = h / (a.n_q_heads / c.n_heads), cap = c.max_pages * c.page_size;
  const uint64_t all = 0xffffffffffffffffull >> (64 - a.n_nodes);
  const uint64_t mask = a.mask ? a.mask[b * a.mask_stride + node] & all : 0;
  const int n = min(max(a.lens[b], 0), cap);
  int lo = 0, end = n;
  if (a.mask) {
    end = mask ? min(cap, n + a.n_nodes) : 0;
    if (a.window) lo = max(0, n + __popcll(mask) - a.window);
  } else if (a.window) {
    lo = max(0, n - a.window);
  }
  constexpr int kPairs = D / 64;
  float2 q[kPairs], o[kPairs];
  const T* qp = (const T*)a.q + b * a.q_seq + node * a.q_node + h * a.q_head;
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    q[i] = load2<T>(qp, 2 * (lane + 32 * i));
    o[i] = make_float2(0.0f, 0.0f);
  }
  const float qscale = a.scale * 1.4426950408889634f;
  float m = -CUDART_INF_F, l = 0.0f;
  for (int p = lo; p < end; ++p) {
    if (p >= n && !((mask >> (p - n)) & 1)) continue;
    const int page = c.table[(int64_t)b * c.table_stride + p / c.page_size];
    if (page < 0 || page >= c.n_pages) continue;
    const int slot = p % c.page_size;
    const int64_t at = kv_page_offset(c, page) + (int64_t)slot * c.slot_stride + hk * c.head_stride;
    float ks = 1.0f, vs = 1.0f;
    if (sizeof(E) == 1) {
      const int64_t s = page * a.sc.page_stride + (int64_t)slot * a.sc.slot_stride + hk * a.sc.head_stride;
      ks = scale_of(a.sc.k[s]);
      vs = scale_of(a.sc.v[s]);
    }
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const float2 k = load2<E>(c.k, at + 2 * (lane + 32 * i));
      s = fmaf(q[i].x, k.x * ks, fmaf(q[i].y, k.y * ks, s));
    }
    for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    s *= qscale;
    const float top = fmaxf(m, s);
    const float f = m == -CUDART_INF_F ? 0.0f : exp2f(m - top);
    const float w = s == -CUDART_INF_F ? 0.0f : exp2f(s - top);
    m = top;
    l = fmaf(l, f, w);
    const float wv = w * vs;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const float2 v = load2<E>(c.v, at + 2 * (lane + 32 * i));
      o[i].x = fmaf(wv, v.x, o[i].x * f);
      o[i].y = fmaf(wv, v.y, o[i].y * f);
    }
    if (vs != vs) l = vs;
  }
  T* out = (T*)a.out + b * a.o_seq + node * a.o_node + h * a.o_head;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int i = 0; i < kPairs; ++i)
    *reinterpret_cast<uint32_t*>(out + 2 * (lane + 32 * i)) = l == 0.0f ? 0u : pack2<T>(o[i].x * inv, o[i].y * inv);
  if (a.lse && lane == 0) a.lse[row] = l == 0.0f ? -CUDART_INF_F : m * 0.69314718f + logf(l);
}

int64_t tree_attn_ws_bytes(const pe_kv_cache&, int, int) { return 256; }

template <typename T, typename E>
static pe_status go(const TreeArgs& a, cudaStream_t st) {
  const int64_t rows = (int64_t)a.c.n_seqs * a.n_nodes * a.n_q_heads;
  const dim3 grid((unsigned)ceil_div(rows, kRowWarps)), block(32 * kRowWarps);
  if (a.c.head_dim == 64)
    PE_TRY_CUDA(launch_pdl(tree_rows_kernel<T, E, 64>, grid, block, 0, st, true, a));
  else if (a.c.head_dim == 128)
    PE_TRY_CUDA(launch_pdl(tree_rows_kernel<T, E, 128>, grid, block, 0, st, true, a));
  else
    PE_TRY_CUDA(launch_pdl(tree_rows_kernel<T, E, 256>, grid, block, 0, st, true, a));
  return PE_OK;
}

pe_status tree_attn_launch(const TreeArgs& a, void*, cudaStream_t st) {
  ProfScope ps(a.mask ? PE_PROF_TREE_ATTN : PE_PROF_DECODE_ATTN, st);
  if (a.dtype == PE_BF16) return a.c.dtype == PE_E4M3 ? go<__nv_bfloat16, uint8_t>(a, st) : go<__nv_bfloat16, __nv_bfloat16>(a, st);
  return a.c.dtype == PE_E4M3 ? go<__half, uint8_t>(a, st) : go<__half, __half>(a, st);
}

}  // namespace pe
