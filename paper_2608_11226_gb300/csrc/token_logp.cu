// Log-probabilities of given tokens with entropy and top alternatives, and
// their gradient (formulas: pe.h).
//
// Forward, one pass over the row: every thread keeps the largest logit m it
// has seen, S = sum e^(scale (x - m)) and T = sum e^(scale (x - m)) (x - m); a
// larger logit rescales them.  Joined over warp, CTA and cluster,
// lse = scale m + ln S and entropy = ln S - scale T / S.  Bound: HBM for
// many rows (an element costs one exponential and about five issue slots, half
// of what the SMs have at the copy rate); for few rows the latency of one
// row, which a cluster of CTAs then shares.
//
// Top alternatives come from the same pass: the k-th largest of the threads'
// maxima bounds the k-th largest logit from below, so only the few threads
// whose maximum reaches it look at their elements again (from L2).
//
// Backward: elementwise from the saved lse and entropy, one read and one write.
#include <cooperative_groups.h>
#include <math_constants.h>

#include "tokens.cuh"

namespace pe {

namespace cg = cooperative_groups;

// Stands for every lower logit and for -inf in the sums (about -1e30, the same
// number in bf16 and fp32): against a row maximum above it their weight is 0.
// A row whose maximum is not above it takes the careful path.
constexpr uint32_t kLowBits = 0xF1490000u;
constexpr float kLog2e = 1.4426950408889634f;

// order-preserving key of a logit: larger logit, larger key; a NaN is the
// largest; equal logits have equal keys (-0 and +0 too); 0 is no key
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

__device__ __forceinline__ float exp_fast(float x) {  // e^x; 0 below -88
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * kLog2e));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {  // NaN if either is
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ float2 both2(float x) { return make_float2(x, x); }

// 16 bytes of a row: kElems elements, read as pairs of fp32
template <typename T> struct Chunk;
template <> struct Chunk<float> {
  static constexpr int kElems = 4, kPairs = 2;
  static constexpr uint32_t kNone = 0xff800000u;  // -inf
  static __device__ __forceinline__ float2 pair(const uint4& v, int i) {
    return i == 0 ? make_float2(__uint_as_float(v.x), __uint_as_float(v.y)) : make_float2(__uint_as_float(v.z), __uint_as_float(v.w));
  }
  template <int U> static __device__ __forceinline__ float largest(const uint4 (&v)[U]) {
    float m = max_nan(max_nan(pair(v[0], 0).x, pair(v[0], 0).y), max_nan(pair(v[0], 1).x, pair(v[0], 1).y));
#pragma unroll
    for (int u = 1; u < U; ++u)
      m = max_nan(m, max_nan(max_nan(pair(v[u], 0).x, pair(v[u], 0).y), max_nan(pair(v[u], 1).x, pair(v[u], 1).y)));
    return m;
  }
  static __device__ __forceinline__ float2 floored(const uint4& v, int i) {
    const float low = __uint_as_float(kLowBits);
    const float2 p = pair(v, i);
    return make_float2(fmaxf(p.x, low), fmaxf(p.y, low));
  }
  static __device__ __forceinline__ void put(uint4& v, int i, float2 p) {
    (i == 0 ? v.x : v.z) = __float_as_uint(p.x);
    (i == 0 ? v.y : v.w) = __float_as_uint(p.y);
  }
};
template <typename T> struct Chunk16 {
  static constexpr int kElems = 8, kPairs = 4;
  static __device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
  static __device__ __forceinline__ void put(uint4& v, int i, float2 p) {
    const uint32_t w = pack2<T>(p.x, p.y);
    (i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w) = w;
  }
};
template <> struct Chunk<__nv_bfloat16> : Chunk16<__nv_bfloat16> {
  static constexpr uint32_t kNone = 0xff80ff80u;
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t y;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
    return y;
  }
  static __device__ __forceinline__ float2 pair(const uint4& v, int i) { return unpack2<__nv_bfloat16>(word(v, i)); }
  static __device__ __forceinline__ float2 floored(const uint4& v, int i) { return unpack2<__nv_bfloat16>(max2(word(v, i), (kLowBits & 0xffff0000u) | (kLowBits >> 16))); }
  template <int U> static __device__ __forceinline__ float largest(const uint4 (&v)[U]) {
    uint32_t m = max2(max2(v[0].x, v[0].y), max2(v[0].z, v[0].w));
#pragma unroll
    for (int u = 1; u < U; ++u) m = max2(m, max2(max2(v[u].x, v[u].y), max2(v[u].z, v[u].w)));
    const float2 p = unpack2<__nv_bfloat16>(m);
    return max_nan(p.x, p.y);
  }
};
template <> struct Chunk<__half> : Chunk16<__half> {
  static constexpr uint32_t kNone = 0xfc00fc00u;
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t y;
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
    return y;
  }
  static __device__ __forceinline__ float2 pair(const uint4& v, int i) { return unpack2<__half>(word(v, i)); }
  static __device__ __forceinline__ float2 floored(const uint4& v, int i) {
    const float low = __uint_as_float(kLowBits);
    const float2 p = pair(v, i);
    return make_float2(fmaxf(p.x, low), fmaxf(p.y, low));
  }
  template <int U> static __device__ __forceinline__ float largest(const uint4 (&v)[U]) {
    uint32_t m = max2(max2(v[0].x, v[0].y), max2(v[0].z, v[0].w));
#pragma unroll
    for (int u = 1; u < U; ++u) m = max2(m, max2(max2(v[u].x, v[u].y), max2(v[u].z, v[u].w)));
    const float2 p = unpack2<__half>(m);
    return max_nan(p.x, p.y);
  }
};

// A row as the 16-byte chunks that hold it: element e lies in chunk
// (e + mis) / kElems.  The first and last chunk may be partly outside the row;
// they are read by element and filled with -inf.
template <typename T> struct Row {
  static constexpr int E = Chunk<T>::kElems;
  const T* x;
  int V, mis;
  __device__ __forceinline__ Row(const T* p, int n) : x(p), V(n), mis((int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T))) {}
  __device__ __forceinline__ int chunks() const { return (int)(((int64_t)mis + V + E - 1) / E); }
  __device__ __forceinline__ int first_whole() const { return mis ? 1 : 0; }
  __device__ __forceinline__ int end_whole() const { return (int)(((int64_t)mis + V) / E); }
  __device__ __forceinline__ uint4 whole(int j) const { return __ldg(reinterpret_cast<const uint4*>(x + ((int64_t)j * E - mis))); }
  // read once, and perhaps written in place: not through the read-only path
  __device__ __forceinline__ uint4 once(int j) const { return __ldcs(reinterpret_cast<const uint4*>(x + ((int64_t)j * E - mis))); }
  __device__ __forceinline__ uint4 any(int j) const {
    if (j >= first_whole() && j < end_whole()) return whole(j);
    alignas(16) T t[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int64_t e = (int64_t)j * E - mis + i;
      t[i] = e >= 0 && e < V ? x[e] : from_f32<T>(-CUDART_INF_F);
    }
    return *reinterpret_cast<const uint4*>(t);
  }
};

// running statistics: the largest logit, S = sum e^(scale (x - m)) and
// T = sum e^(scale (x - m)) (x - m).  Differences first, so that logits of any
// size leave them at or below 0.
struct Stat {
  float m, S, T;
};

__device__ __forceinline__ void rebase(Stat& s, float m, float scale) {  // to the larger m (or NaN)
  const float d = fmaxf(s.m - m, -200.0f / scale);  // e^-200 is 0 and keeps 0 * d finite
  const float f = m != m ? m : exp_fast(d * scale);
  s.T = f * fmaf(s.S, d, s.T);
  s.S *= f;
  s.m = m;
}
__device__ __forceinline__ void join(Stat& a, Stat b, float scale) {
  const float m = max_nan(a.m, b.m);
  rebase(a, m, scale);
  rebase(b, m, scale);
  a.S += b.S;
  a.T += b.T;
}

template <typename T, int U>
__device__ __forceinline__ void absorb(const uint4 (&v)[U], float scale, Stat& s) {
  using C = Chunk<T>;
  const float cm = max_nan(C::largest(v), s.m);
  if (cm != s.m) rebase(s, cm, scale);
  const float2 m = both2(-s.m), l2 = both2(scale * kLog2e);
  float2 S = make_float2(s.S, 0.0f), Ts = make_float2(s.T, 0.0f);
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < C::kPairs; ++i) {
      const float2 d = __fadd2_rn(C::floored(v[u], i), m);
      const float2 a = __fmul2_rn(d, l2);
      float2 e;
      asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(a.x));
      asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(a.y));
      S = __fadd2_rn(S, e);
      Ts = __ffma2_rn(e, d, Ts);
    }
  s.S = S.x + S.y;
  s.T = Ts.x + Ts.y;
}

// ---------------------------------------------------------------------------
// top alternatives: keys (order_key, ~index), largest first, in the lanes of a warp
// ---------------------------------------------------------------------------
using Key = unsigned long long;
__device__ __forceinline__ Key make_key(float x, int e) { return ((Key)order_key(x) << 32) | (0xffffffffu - (uint32_t)e); }

__device__ __forceinline__ Key exchange(Key k, int x, bool keep_large) {
  const Key o = __shfl_xor_sync(0xffffffffu, k, x);
  return (k > o) == keep_large ? k : o;
}
__device__ __forceinline__ Key sort_desc(Key k) {  // bitonic, 32 lanes
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
    for (int x = size / 2; x; x >>= 1) k = exchange(k, x, ((lane & x) == 0) == ((lane & size) == 0 || size == 32));
  return k;
}
// the 32 largest of two descending lists, descending
__device__ __forceinline__ Key merge_desc(Key a, Key b) {
  const int lane = threadIdx.x & 31;
  const Key r = __shfl_sync(0xffffffffu, b, 31 - lane);
  a = a > r ? a : r;
#pragma unroll
  for (int x = 16; x; x >>= 1) a = exchange(a, x, (lane & x) == 0);
  return a;
}

constexpr int kCand = 512;  // candidates held for sorting

template <int THREADS> struct LogpShared {
  float m[THREADS / 32], S[THREADS / 32], T[THREADS / 32];
  Stat slice;          // of this CTA's part of the row
  Key top[32];
  Key cand[kCand];
  int count;
  uint32_t part[THREADS / 32];
  Key best;
};

// counts over the CTA
template <int THREADS> __device__ __forceinline__ int count_block(bool p) {
  return THREADS == 32 ? __popc(__ballot_sync(0xffffffffu, p)) : __syncthreads_count(p);
}
template <int THREADS> __device__ __forceinline__ void sync_block() {
  if (THREADS == 32)
    __syncwarp();
  else
    __syncthreads();
}

// The k largest keys of chunks [j0, j1) into sh.top (missing ones 0).  mine:
// the largest logit of this thread's chunks j0 + tid + i * THREADS.
template <typename T, int THREADS>
__device__ void top_slice(const Row<T>& row, int j0, int j1, float mine, int k, LogpShared<THREADS>& sh) {
  using C = Chunk<T>;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool has = j0 + tid < j1;
  // the upper 16 bits of the k-th largest thread maximum, bit by bit: a bound
  // from below that at least k elements reach, or 0 where fewer threads have any
  const uint32_t my = has ? order_key(mine) : 0u;
  uint32_t tau = 0;
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t t = tau | (1u << bit);
    if (count_block<THREADS>(my >= t) >= k) tau = t;
  }
  // the elements that reach it
  auto collect = [&](uint32_t least) {
    if (tid == 0) sh.count = 0;
    sync_block<THREADS>();
    uint32_t who = __ballot_sync(0xffffffffu, has && my >= least);
    while (who) {
      const int l = __ffs(who) - 1;
      who &= who - 1;
      for (int64_t j = (int64_t)j0 + warp * 32 + l + (int64_t)lane * THREADS; j < j1; j += 32 * (int64_t)THREADS) {
        if (*(volatile int*)&sh.count > kCand) break;  // too many already: how many does not matter
        const uint4 v = row.any((int)j);
#pragma unroll
        for (int i = 0; i < C::kPairs; ++i) {
          const float2 p = C::pair(v, i);
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float z = y ? p.y : p.x;
            const int64_t e = (int64_t)j * C::kElems - row.mis + 2 * i + y;
            if (order_key(z) >= least && e >= 0 && e < row.V) {
              const int at = atomicAdd(&sh.count, 1);
              if (at < kCand) sh.cand[at] = make_key(z, (int)e);
            }
          }
        }
      }
    }
    sync_block<THREADS>();
    const int n = sh.count;
    sync_block<THREADS>();
    return n;
  };
  // keys from `least` on are collected, then sorted; the rest is found below.
  // A bound at the stand-in for low logits says nothing: a thread's maximum is
  // at least that
  const uint32_t low = order_key(__uint_as_float(kLowBits));
  const bool every = (int64_t)(j1 - j0) * C::kElems <= kCand;
  uint32_t least = every ? 0u : tau > low ? tau : low + 1;
  int n = collect(least);
  if (n > kCand && least == tau) n = collect(++least);  // ties at the bound
  bool inclusive = false;
  if (n > kCand) {  // a row that crowds its large logits into few threads
    n = 0;
    least = 0xffffffffu;
    inclusive = true;
  }
  // sorted by one warp, 32 at a time; the order in which they came does not matter
  if (warp == 0) {
    Key top = 0;
    for (int i = 0; i < n; i += 32) {
      const Key c = sort_desc(i + lane < n ? sh.cand[i + lane] : 0);
      top = i ? merge_desc(top, c) : c;
    }
    sh.top[lane] = lane < k ? top : 0;
  }
  // What is left is found value by value: the largest key below the last one,
  // then its elements from the lowest index on.  A row with fewer than k
  // allowed tokens needs one such round, for -inf.
  uint32_t below = least;
  int filled = min(n, k);
  while (filled < k && !every) {
    if (tid == 0) sh.best = 0;
    sync_block<THREADS>();
    uint32_t best = 0;
    for (int64_t j = (int64_t)j0 + tid; j < j1; j += THREADS) {
      const uint4 v = row.any((int)j);
#pragma unroll
      for (int i = 0; i < C::kElems; ++i) {
        const int64_t e = j * C::kElems - row.mis + i;
        const float2 p = C::pair(v, i / 2);
        const uint32_t q = order_key(i & 1 ? p.y : p.x);
        if (e >= 0 && e < row.V && (q < below || inclusive)) best = max(best, q);
      }
    }
    atomicMax(&sh.best, (Key)best);
    sync_block<THREADS>();
    best = (uint32_t)sh.best;
    inclusive = false;
    below = best;
    if (best == 0) break;  // the slice is used up
    for (int64_t jj = j0; jj < j1 && filled < k; jj += THREADS) {
      const int64_t j = jj + tid;
      uint32_t hit = 0;
      if (j < j1) {
        const uint4 v = row.any((int)j);
#pragma unroll
        for (int i = 0; i < C::kElems; ++i) {
          const int64_t e = j * C::kElems - row.mis + i;
          const float2 p = C::pair(v, i / 2);
          if (e >= 0 && e < row.V && order_key(i & 1 ? p.y : p.x) == best) hit |= 1u << i;
        }
      }
      uint32_t before = __popc(hit);
      for (int x = 1; x < 32; x <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, before, x);
        if (lane >= x) before += y;
      }
      if (lane == 31) sh.part[warp] = before;
      sync_block<THREADS>();
      uint32_t base = 0, all = 0;
      for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) base += sh.part[w];
        all += sh.part[w];
      }
      int at = filled + (int)(base + before - __popc(hit));
      for (; hit && at < k; hit &= hit - 1, ++at)
        sh.top[at] = ((Key)best << 32) | (0xffffffffu - (uint32_t)(j * C::kElems - row.mis + __ffs(hit) - 1));
      filled = (int)min((int64_t)k, (int64_t)filled + all);
      sync_block<THREADS>();
    }
  }
}

// A row is cut into gridDim.x slices, one for each CTA of its cluster.
template <typename T, int THREADS, bool TOP>
__global__ void __launch_bounds__(THREADS) token_logp_kernel(LogpArgs a) {
  constexpr int U = 4, kWarps = THREADS / 32;
  __shared__ LogpShared<THREADS> sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = blockIdx.x, ranks = gridDim.x;
  const int64_t r = blockIdx.y + (int64_t)blockIdx.z * gridDim.y;
  if (r >= a.n) return;  // a whole cluster, or none of it
  const Row<T> row((const T*)a.logits + r * a.row_stride, a.V);
  const int all = row.chunks();
  const int j0 = (int)((int64_t)all * rank / ranks), j1 = (int)((int64_t)all * (rank + 1) / ranks);
  const int w0 = row.first_whole(), w1 = min(j1, row.end_whole());
  // the target's logit, on its way while the row is read
  int t = -1;
  float zt = 0.0f;
  if (rank == 0 && tid == 0 && a.logp) {
    t = a.tokens[r];
    if (t >= 0 && t < a.V) zt = to_f32(row.x[t]);
  }

  Stat s;
  s.m = __uint_as_float(kLowBits);
  s.S = s.T = 0.0f;
  for (int64_t j = j0; j < j1; j += U * THREADS) {
    uint4 v[U];
    if (j >= w0 && j + U * THREADS <= w1) {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = row.whole((int)j + u * THREADS + tid);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t jj = j + u * THREADS + tid;
        v[u] = jj < j1 ? row.any((int)jj) : make_uint4(Chunk<T>::kNone, Chunk<T>::kNone, Chunk<T>::kNone, Chunk<T>::kNone);
      }
    }
    absorb<T, U>(v, a.scale, s);
  }
  const float mine = s.m;
#pragma unroll
  for (int x = 16; x; x >>= 1) {
    Stat o;
    o.m = __shfl_xor_sync(0xffffffffu, s.m, x);
    o.S = __shfl_xor_sync(0xffffffffu, s.S, x);
    o.T = __shfl_xor_sync(0xffffffffu, s.T, x);
    join(s, o, a.scale);
  }
  if (kWarps > 1) {
    if (lane == 0) {
      sh.m[warp] = s.m;
      sh.S[warp] = s.S;
      sh.T[warp] = s.T;
    }
    __syncthreads();
    s = Stat{sh.m[0], sh.S[0], sh.T[0]};
#pragma unroll
    for (int w = 1; w < kWarps; ++w) join(s, Stat{sh.m[w], sh.S[w], sh.T[w]}, a.scale);
  }
  if (TOP) top_slice<T, THREADS>(row, j0, j1, mine, a.top_k, sh);
  Key top = 0;
  if (ranks > 1) {
    cg::cluster_group cl = cg::this_cluster();
    if (tid == 0) sh.slice = s;
    cl.sync();
    if (rank == 0) {
      for (int p = 1; p < ranks; ++p) join(s, *cl.map_shared_rank(&sh.slice, p), a.scale);
      if (TOP && warp == 0) {
        top = sh.top[lane];
        for (int p = 1; p < ranks; ++p) top = merge_desc(top, cl.map_shared_rank(sh.top, p)[lane]);
      }
    }
    cl.sync();  // the others' shared memory has been read
    if (rank) return;
  } else if (TOP) {
    sync_block<THREADS>();
    if (warp == 0) top = sh.top[lane];
  }

  if (s.m <= __uint_as_float(kLowBits)) {
    // nothing above the stand-in: -inf alone, or masks of the type's lowest
    // value alone; by the definition, element by element
    float m = -CUDART_INF_F;
    for (int e = tid; e < a.V; e += THREADS) m = fmaxf(m, to_f32(row.x[e]));
    for (int x = 16; x; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
    sync_block<THREADS>();
    if (lane == 0) sh.m[warp] = m;
    sync_block<THREADS>();
    for (int w = 0; w < kWarps; ++w) m = fmaxf(m, sh.m[w]);
    s.m = m;
    float S = 0.0f, D = 0.0f;
    if (m != -CUDART_INF_F)
      for (int e = tid; e < a.V; e += THREADS) {
        const float d = to_f32(row.x[e]) - m;
        const float p = exp_fast(d * a.scale);
        S += p;
        D += p == 0.0f ? 0.0f : p * d;
      }
    for (int x = 16; x; x >>= 1) {
      S += __shfl_xor_sync(0xffffffffu, S, x);
      D += __shfl_xor_sync(0xffffffffu, D, x);
    }
    if (lane == 0) {
      sh.S[warp] = S;
      sh.T[warp] = D;
    }
    sync_block<THREADS>();
    s.S = s.T = 0.0f;
    for (int w = 0; w < kWarps; ++w) {
      s.S += sh.S[w];
      s.T += sh.T[w];
    }
  }
  const bool empty = s.m == -CUDART_INF_F;
  const float ln = logf(s.S);
  if (tid == 0) {
    if (a.lse) a.lse[r] = empty ? -CUDART_INF_F : fmaf(s.m, a.scale, ln);
    if (a.entropy) a.entropy[r] = empty ? 0.0f : ln - a.scale * s.T / s.S;
    if (a.logp) a.logp[r] = t < 0 || t >= a.V ? 0.0f : empty ? -CUDART_INF_F : (zt - s.m) * a.scale - ln;
  }
  if (TOP && tid < a.top_k) {
    a.top_id[r * a.top_k + tid] = (int32_t)(0xffffffffu - (uint32_t)top);
    a.top_logp[r * a.top_k + tid] = empty ? -CUDART_INF_F : (key_logit((uint32_t)(top >> 32)) - s.m) * a.scale - ln;
  }
}

// ---------------------------------------------------------------------------
// gradient: THREADS threads on kGradChunks chunks each of one row
// ---------------------------------------------------------------------------
constexpr int kGradChunks = 4;

template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS) token_logp_grad_kernel(LogpGradArgs a) {
  using C = Chunk<T>;
  const int64_t r = blockIdx.y + (int64_t)blockIdx.z * gridDim.y;
  if (r >= a.n) return;
  const Row<T> row((const T*)a.logits + r * a.row_stride, a.V);
  T* y = (T*)a.dlogits + r * a.d_row_stride;
  const int64_t j = (int64_t)blockIdx.x * (kGradChunks * THREADS) + threadIdx.x;
  const int all = row.chunks(), w0 = row.first_whole(), w1 = row.end_whole();
  if (j >= all) return;
  uint4 v[kGradChunks];
#pragma unroll
  for (int u = 0; u < kGradChunks; ++u) {
    const int64_t c = j + u * THREADS;
    if (c >= w0 && c < w1) v[u] = row.once((int)c);
  }
  const float lse = a.lse[r];
  const int t = a.g_logp ? a.tokens[r] : -1;
  const float g = t >= 0 && t < a.V ? a.g_logp[r] : 0.0f;
  const float ge = a.g_entropy ? a.g_entropy[r] : 0.0f, H = a.g_entropy ? a.entropy[r] : 0.0f;
  // dz = p (A + B ln p)
  const float A = -a.scale * fmaf(ge, H, g), B = -a.scale * ge;
  const bool empty = lse == -CUDART_INF_F;
  const bool same = ((reinterpret_cast<uintptr_t>(row.x) ^ reinterpret_cast<uintptr_t>(y)) & 15) == 0;
  const float2 sc = both2(a.scale), L = both2(-lse), l2 = both2(kLog2e), A2 = both2(A), B2 = both2(B);
#pragma unroll
  for (int u = 0; u < kGradChunks; ++u) {
    const int64_t c = j + u * THREADS;
    if (c >= all) break;
    const bool whole = c >= w0 && c < w1;
    const uint4 in = whole ? v[u] : row.any((int)c);
    uint4 out;
#pragma unroll
    for (int i = 0; i < C::kPairs; ++i) {
      float2 d = __ffma2_rn(C::pair(in, i), sc, L);
      // ln p of a forbidden token, kept finite: p is 0 there.  NaN stays
      d.x = d.x < -1000.0f ? -1000.0f : d.x;
      d.y = d.y < -1000.0f ? -1000.0f : d.y;
      const float2 x = __fmul2_rn(d, l2);
      float2 p;
      asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(p.x) : "f"(x.x));
      asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(p.y) : "f"(x.y));
      float2 z = __fmul2_rn(p, __ffma2_rn(B2, d, A2));
      const int e = (int)(c * C::kElems - row.mis) + 2 * i;
      if (e == t) z.x = fmaf(a.scale, g, z.x);  // the target's own term
      if (e + 1 == t) z.y = fmaf(a.scale, g, z.y);
      if (empty) z = both2(0.0f);
      C::put(out, i, z);
    }
    if (whole && same) {
      __stcs(reinterpret_cast<uint4*>(y + (c * C::kElems - row.mis)), out);
    } else {
      alignas(16) T e[C::kElems];
      *reinterpret_cast<uint4*>(e) = out;
#pragma unroll
      for (int i = 0; i < C::kElems; ++i) {
        const int64_t at = c * C::kElems - row.mis + i;
        if (at >= 0 && at < a.V) y[at] = e[i];
      }
    }
  }
}

// rows of a grid: y, and z beyond its limit
static dim3 row_grid(int x, int64_t n) {
  const int64_t y = n < 65535 ? n : 65535;
  return dim3(x, (unsigned)y, (unsigned)((n + y - 1) / y));
}

template <typename T, int THREADS>
static pe_status go_logp(const LogpArgs& a, int ranks, cudaStream_t st) {
  auto kern = a.top_k ? token_logp_kernel<T, THREADS, true> : token_logp_kernel<T, THREADS, false>;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = ranks;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cudaLaunchConfig_t lc{};
  lc.gridDim = row_grid(ranks, a.n);
  lc.blockDim = THREADS;
  lc.stream = st;
  lc.attrs = &at;
  lc.numAttrs = ranks > 1 ? 1 : 0;
  PE_TRY_CUDA(cudaLaunchKernelEx(&lc, kern, a));
  return PE_OK;
}

template <typename T>
static pe_status logp(const LogpArgs& a, cudaStream_t st) {
  const int64_t chunks = ceil_div(a.V, Chunk<T>::kElems);
  // a CTA of a row as wide as the row gives each thread eight chunks
  if (chunks <= 8 * 32) return go_logp<T, 32>(a, 1, st);
  if (chunks <= 8 * 128) return go_logp<T, 128>(a, 1, st);
  // few rows: a cluster shares one, while each thread has four chunks
  int ranks = 1;
  while (ranks < 8 && a.n * ranks * 2 <= 304 && chunks >= 512 * 4 * ranks * 2) ranks *= 2;
  return go_logp<T, 512>(a, ranks, st);
}

template <typename T, int THREADS>
static void go_grad(const LogpGradArgs& a, int64_t chunks, cudaStream_t st) {
  token_logp_grad_kernel<T, THREADS><<<row_grid(ceil_div(chunks, kGradChunks * THREADS), a.n), THREADS, 0, st>>>(a);
}

template <typename T>
static void grad(const LogpGradArgs& a, cudaStream_t st) {
  const int64_t chunks = (int64_t)ceil_div(a.V, Chunk<T>::kElems) + 1;  // one more where the row is not aligned
  if (chunks <= 4 * 32)
    go_grad<T, 32>(a, chunks, st);
  else
    go_grad<T, 256>(a, chunks, st);
}

pe_status token_logp_launch(const LogpArgs& a, int dtype, cudaStream_t st) {
  ProfScope ps(PE_PROF_TOKEN_LOGP, st);
  if (dtype == PE_F32) return logp<float>(a, st);
  if (dtype == PE_BF16) return logp<__nv_bfloat16>(a, st);
  return logp<__half>(a, st);
}

pe_status token_logp_grad_launch(const LogpGradArgs& a, int dtype, cudaStream_t st) {
  ProfScope ps(PE_PROF_TOKEN_LOGP_GRAD, st);
  if (dtype == PE_F32)
    grad<float>(a, st);
  else if (dtype == PE_BF16)
    grad<__nv_bfloat16>(a, st);
  else
    grad<__half>(a, st);
  PE_CHECK_LAUNCH("token_logp_grad");
  return PE_OK;
}

}  // namespace pe
