// Shared parts of the token operators (kv_append.cu, decode_attn.cu,
// token_logp.cu; their C entry points are in token_api.cu).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace pe {

// Every kernel of these operators is launched programmatically: it may be set
// up while the kernel ahead in the stream drains, and waits for that one's end
// (pdl_enter) before it touches memory.  Back to back that saves about 2 us of a
// pass (append of 4,001 tokens 14.4 to 12.2 us, gradient of 333 x 32,003 16.4 to
// 14.4, one row's log-probabilities 10.2 to 7.3).

// element <-> fp32 (one rounding to nearest even on the way out)
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

// two elements in a word, the first in the low half
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

// element offset of (page, slot 0, head 0), 64-bit: a cache of 2^31 elements
// is 4 GB per tensor
__device__ __forceinline__ int64_t kv_page_offset(const pe_kv_cache& c, int page) { return (int64_t)page * c.page_stride; }

struct DecodeArgs {
  pe_kv_cache c;
  const void* q;
  void* out;
  float* lse;
  const int32_t* lens;
  int64_t q_seq, q_head, o_seq, o_head;
  float scale;
  int32_t n_q_heads, window;
};

struct LogpArgs {
  const void* logits;
  const int32_t* tokens;
  float *logp, *entropy, *lse, *top_logp;
  int32_t* top_id;
  int64_t n, row_stride;
  int32_t V, top_k;
  float scale;
};

struct LogpGradArgs {
  const void* logits;
  void* dlogits;
  const int32_t* tokens;
  const float *lse, *entropy, *g_logp, *g_entropy;
  int64_t n, row_stride, d_row_stride;
  int32_t V;
  float scale;
};

pe_status kv_append_launch(const pe_kv_cache& c, const pe_kv_tokens& t, cudaStream_t st);
int64_t decode_attn_ws_bytes(const pe_kv_cache& c, int n_q_heads);
pe_status decode_attn_launch(const DecodeArgs& a, void* ws, cudaStream_t st);
pe_status token_logp_launch(const LogpArgs& a, int dtype, cudaStream_t st);
pe_status token_logp_grad_launch(const LogpGradArgs& a, int dtype, cudaStream_t st);

}  // namespace pe
