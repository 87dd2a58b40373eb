// Log-probabilities of given tokens with entropy and top alternatives, and
// their gradient (formulas: pe.h).  One CTA per row.
#include <math_constants.h>

#include "tokens.cuh"

namespace pe {

constexpr int kRowThreads = 256;

// order-preserving key of a logit: larger logit, larger key; a NaN is the
// largest; equal logits compare equal (-0 and +0 too)
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <typename F>
__device__ __forceinline__ float block_reduce(float v, F f, float* sh) {
  for (int x = 16; x; x >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, x));
  __syncthreads();
  if (threadIdx.x % 32 == 0) sh[threadIdx.x / 32] = v;
  __syncthreads();
  v = sh[0];
  for (int i = 1; i < kRowThreads / 32; ++i) v = f(v, sh[i]);
  return v;
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) token_logp_kernel(LogpArgs a) {
  __shared__ float sh[kRowThreads / 32];
  __shared__ unsigned long long best;
  const int64_t r = blockIdx.x;
  const T* x = (const T*)a.logits + r * a.row_stride;
  float m = -CUDART_INF_F;
  bool nan = false;
  for (int j = threadIdx.x; j < a.V; j += kRowThreads) {
    const float z = to_f32(x[j]) * a.scale;
    nan |= z != z;
    m = fmaxf(m, z);
  }
  auto mx = [](float p, float q) { return fmaxf(p, q); };
  auto add = [](float p, float q) { return p + q; };
  m = block_reduce(m, mx, sh);
  if (__syncthreads_or(nan)) m = CUDART_NAN_F;
  float S = 0.0f, D = 0.0f;
  const bool empty = m == -CUDART_INF_F;
  if (!empty)
    for (int j = threadIdx.x; j < a.V; j += kRowThreads) {
      const float d = to_f32(x[j]) * a.scale - m;
      if (d == -CUDART_INF_F) continue;
      const float e = expf(d);
      S += e;
      D += e * d;
    }
  S = block_reduce(S, add, sh);
  D = block_reduce(D, add, sh);
  const float ln = logf(S);
  if (threadIdx.x == 0) {
    if (a.lse) a.lse[r] = empty ? -CUDART_INF_F : m + ln;
    if (a.entropy) a.entropy[r] = empty ? 0.0f : ln - D / S;
    if (a.logp) {
      const int t = a.tokens[r];
      const bool has = t >= 0 && t < a.V;
      a.logp[r] = !has ? 0.0f : empty ? -CUDART_INF_F : (to_f32(x[t]) * a.scale - m) - ln;
    }
  }
  unsigned long long last = ~0ull;
  for (int k = 0; k < a.top_k; ++k) {
    unsigned long long mine = 0;
    for (int j = threadIdx.x; j < a.V; j += kRowThreads) {
      const unsigned long long key = ((unsigned long long)order_key(to_f32(x[j])) << 32) | (0xffffffffu - (uint32_t)j);
      if (key < last && key > mine) mine = key;
    }
    __syncthreads();
    if (threadIdx.x == 0) best = 0;
    __syncthreads();
    atomicMax(&best, mine);
    __syncthreads();
    last = best;
    if (threadIdx.x == 0) {
      const uint32_t id = 0xffffffffu - (uint32_t)last;
      a.top_id[r * a.top_k + k] = (int32_t)id;
      a.top_logp[r * a.top_k + k] = empty ? -CUDART_INF_F : (to_f32(x[id]) * a.scale - m) - ln;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) token_logp_grad_kernel(LogpGradArgs a) {
  const int64_t r = blockIdx.x;
  const T* x = (const T*)a.logits + r * a.row_stride;
  T* y = (T*)a.dlogits + r * a.d_row_stride;
  const float lse = a.lse[r];
  const int t = a.g_logp ? a.tokens[r] : -1;
  const float g = t >= 0 && t < a.V ? a.g_logp[r] : 0.0f;
  const float ge = a.g_entropy ? a.g_entropy[r] : 0.0f, H = a.g_entropy ? a.entropy[r] : 0.0f;
  for (int j = threadIdx.x; j < a.V; j += kRowThreads) {
    const float d = to_f32(x[j]) * a.scale - lse;
    float z = 0.0f;
    if (d != -CUDART_INF_F) {
      const float p = expf(d);
      z = -p * (g + ge * (d + H));
    }
    z *= a.scale;
    if (j == t) z = fmaf(a.scale, g, z);  // the target's own term rounded once
    y[j] = from_f32<T>(lse == -CUDART_INF_F ? 0.0f : z);
  }
}

pe_status token_logp_launch(const LogpArgs& a, int dtype, cudaStream_t st) {
  ProfScope ps(PE_PROF_TOKEN_LOGP, st);
  const unsigned grid = (unsigned)a.n;
  if (dtype == PE_F32)
    token_logp_kernel<float><<<grid, kRowThreads, 0, st>>>(a);
  else if (dtype == PE_BF16)
    token_logp_kernel<__nv_bfloat16><<<grid, kRowThreads, 0, st>>>(a);
  else
    token_logp_kernel<__half><<<grid, kRowThreads, 0, st>>>(a);
  PE_CHECK_LAUNCH("token_logp");
  return PE_OK;
}

pe_status token_logp_grad_launch(const LogpGradArgs& a, int dtype, cudaStream_t st) {
  ProfScope ps(PE_PROF_TOKEN_LOGP_GRAD, st);
  const unsigned grid = (unsigned)a.n;
  if (dtype == PE_F32)
    token_logp_grad_kernel<float><<<grid, kRowThreads, 0, st>>>(a);
  else if (dtype == PE_BF16)
    token_logp_grad_kernel<__nv_bfloat16><<<grid, kRowThreads, 0, st>>>(a);
  else
    token_logp_grad_kernel<__half><<<grid, kRowThreads, 0, st>>>(a);
  PE_CHECK_LAUNCH("token_logp_grad");
  return PE_OK;
}

}  // namespace pe
