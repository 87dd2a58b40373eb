// Log-probabilities of given tokens with entropy and top alternatives, and
// their gradient (formulas: pe.h).
//
// Forward, one pass over the row: every thread keeps the largest logit m it
// has seen, S = sum e^(scale (x - m)) and T = sum e^(scale (x - m)) (x - m); a
// larger logit rescales them.  Joined over warp, CTA and cluster,
// lse = scale m + ln S and entropy = ln S - scale T / S.  Bound: HBM for
// many rows (an element costs one exponential and about five issue slots, half
// of what the SMs have at the copy rate); for few rows the latency of one
// row, which a cluster of CTAs then shares.  CTAs, or warps where a row is
// short, go through rows and have the next row's first loads on their way
// while they join the sums of one.
//
// Top alternatives come from the same pass: the k-th largest of 32 maxima, each
// of some threads' elements, bounds the k-th largest logit from below, so only
// the few threads whose maximum reaches it look at their elements again (from L2).
//
// Backward: elementwise from the saved lse and entropy, one read and one write.
// Rows of the gradient that lie otherwise to 16 bytes than the logits' are stored
// element by element (4,096 x 32,003 in bf16: 303 us for 90).
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

// e^x within 2^-22 + 2^-24 |x|; 0 below -88.  Against 64 bits, 8,192 rows of
// 131,072 bf16 logits are off by 8.3e-8 in all, elementary fp32 operations by 5.8e-8.
__device__ __forceinline__ float exp_fast(float x) {
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
  static __device__ __forceinline__ float at(const uint4& v, int i) { return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w); }
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
  static __device__ __forceinline__ float at(const uint4& v, int i) {
    const float2 p = unpack2<T>(word(v, i >> 1));
    return i & 1 ? p.y : p.x;
  }
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
  // coherent: the kernel may be set up before the one that writes the logits has ended
  __device__ __forceinline__ uint4 whole(int j) const { return __ldcg(reinterpret_cast<const uint4*>(x + ((int64_t)j * E - mis))); }
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
// over the first N lanes of each group of N lanes
template <int N> __device__ __forceinline__ void join_lanes(Stat& s, float scale) {
  float m = s.m;
#pragma unroll
  for (int x = N / 2; x; x >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, x));
  rebase(s, m, scale);
#pragma unroll
  for (int x = N / 2; x; x >>= 1) {
    s.S += __shfl_xor_sync(0xffffffffu, s.S, x);
    s.T += __shfl_xor_sync(0xffffffffu, s.T, x);
  }
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

// what the threads of a row share
template <int ROWT, bool TOP> struct RowShared {
  static constexpr int kWarps = ROWT / 32, kCand = !TOP ? 1 : ROWT == 32 ? 256 : 512;  // candidates held for sorting
  Stat warp[2][kWarps];  // of the warps; rows take turns
  Stat slice;            // of a rank's part of the row
  Key top[32];
  Key cand[kCand];
  Key best;
  uint32_t most[32];     // the warps' largest maxima
  uint32_t part[kWarps];
  int count;
  uint8_t who[kWarps][32];
};

template <int ROWT> __device__ __forceinline__ void sync_row() {
  if (ROWT == 32)
    __syncwarp();
  else
    __syncthreads();
}

// The k largest keys of chunks [j0, j1) into sh.top (missing ones 0).  mine:
// the largest logit of this thread's chunks j0 + tid + i * ROWT.
template <typename T, int ROWT>
__device__ void top_slice(const Row<T>& row, int j0, int j1, float mine, int k, RowShared<ROWT, true>& sh) {
  using C = Chunk<T>;
  constexpr int kWarps = ROWT / 32, kCand = RowShared<ROWT, true>::kCand;
  const int tid = threadIdx.x % ROWT, lane = tid & 31, warp = tid / 32;
  const bool has = j0 + tid < j1;
  const uint32_t my = has ? order_key(mine) : 0u;
  // 32 thread maxima, the largest 32 / kWarps of each warp: at least k elements
  // reach their k-th largest
  uint32_t m = my;
  if (kWarps > 1) {
    uint32_t v = my;
#pragma unroll
    for (int i = 0; i < 32 / kWarps; ++i) {
      const uint32_t best = __reduce_max_sync(0xffffffffu, v);
      if (lane == 0) sh.most[warp * (32 / kWarps) + i] = best;
      if (lane == __ffs(__ballot_sync(0xffffffffu, v == best)) - 1) v = 0;
    }
    if (tid == 0) sh.count = 0;
    __syncthreads();
    m = sh.most[lane];
  } else {
    if (lane == 0) sh.count = 0;
    __syncwarp();
  }
  int above = 0;  // maxima that come before this lane's
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const uint32_t o = __shfl_sync(0xffffffffu, m, i);
    above += o > m || (o == m && i < lane);
  }
  const uint32_t tau = __shfl_sync(0xffffffffu, m, __ffs(__ballot_sync(0xffffffffu, above == k - 1)) - 1);

  const bool every = (int64_t)(j1 - j0) * C::kElems <= kCand;  // the candidates hold the slice
  // the elements that reach `least`: a warp goes through the chunks of its
  // threads that have any
  const int per = (j1 - j0 + ROWT - 1) / ROWT;
  auto collect = [&](uint32_t least) {
    const uint32_t who = __ballot_sync(0xffffffffu, has && my >= least);
    const float bound = key_logit(least);  // 0 becomes NaN, which nothing is below
    if ((who >> lane) & 1) sh.who[warp][__popc(who & ((1u << lane) - 1))] = (uint8_t)lane;
    __syncwarp();
    const int pairs = __popc(who) * per;
    for (int p0 = 0; p0 < pairs; p0 += 64) {  // the warp stays together: all its branches are taken by all lanes
      // Too many already: how many does not matter.  Other warps change the
      // count, so one lane reads it for all: lanes that saw different counts
      // would part, and the warp's collectives below wait for every lane.
      int seen = 0;
      if (lane == 0) seen = *(volatile int*)&sh.count;
      if (__shfl_sync(0xffffffffu, seen, 0) > kCand) break;
      uint4 v[2];
      int64_t e[2];
      uint32_t hit[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int p = p0 + 32 * u + lane, q = p / per;
        const int64_t j = (int64_t)j0 + warp * 32 + sh.who[warp][q & 31] + (int64_t)(p - q * per) * ROWT;
        const bool in = p < pairs && j < j1;
        v[u] = in ? row.any((int)j) : make_uint4(0, 0, 0, 0);
        e[u] = j * C::kElems - row.mis;  // of the chunk's first element
        const int64_t lo = max(-e[u], (int64_t)0), hi = min(row.V - e[u], (int64_t)C::kElems);  // elements of the row
        hit[u] = in && hi > lo ? ((1u << hi) - 1) & ~((1u << lo) - 1) : 0u;
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        uint32_t least_hit = 0;
#pragma unroll
        for (int i = 0; i < C::kPairs; ++i) {
          const float2 z = C::pair(v[u], i);
          least_hit |= (z.x < bound ? 0u : 1u << (2 * i)) | (z.y < bound ? 0u : 2u << (2 * i));  // a NaN is the highest
        }
        hit[u] &= least_hit;
        for (uint32_t any; (any = __ballot_sync(0xffffffffu, hit[u] != 0)) != 0; hit[u] &= hit[u] - 1) {
          int base = 0;
          if (lane == 0) base = atomicAdd(&sh.count, __popc(any));
          base = __shfl_sync(0xffffffffu, base, 0);
          const int i = __ffs(hit[u]) - 1, at = base + __popc(any & ((1u << lane) - 1));
          if (hit[u] && at < kCand) sh.cand[at] = make_key(C::at(v[u], i), (int)(e[u] + i));
        }
      }
    }
    sync_row<ROWT>();
    return sh.count;
  };
  // keys from `least` on are collected, then sorted; the rest is found below.
  // A bound at the stand-in for low logits says nothing: a thread's maximum is
  // at least that
  const uint32_t low = order_key(__uint_as_float(kLowBits));
  uint32_t least = every ? 0u : tau > low ? tau : low + 1;
  int n = collect(least);
  if (n > kCand && least == tau) {  // ties at the bound
    sync_row<ROWT>();
    if (tid == 0) sh.count = 0;
    sync_row<ROWT>();
    n = collect(++least);
  }
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
    sync_row<ROWT>();
    uint32_t best = 0;
    for (int64_t j = (int64_t)j0 + tid; j < j1; j += ROWT) {
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
    sync_row<ROWT>();
    best = (uint32_t)sh.best;
    inclusive = false;
    below = best;
    if (best == 0) break;  // the slice is used up
    for (int64_t jj = j0; jj < j1 && filled < k; jj += ROWT) {
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
      sync_row<ROWT>();
      uint32_t base = 0, all = 0;
      for (int w = 0; w < kWarps; ++w) {
        if (w < warp) base += sh.part[w];
        all += sh.part[w];
      }
      int at = filled + (int)(base + before - __popc(hit));
      for (; hit && at < k; hit &= hit - 1, ++at)
        sh.top[at] = ((Key)best << 32) | (0xffffffffu - (uint32_t)(j * C::kElems - row.mis + __ffs(hit) - 1));
      filled = (int)min((int64_t)k, (int64_t)filled + all);
      sync_row<ROWT>();
    }
  }
}

// nothing above the stand-in: -inf alone, or masks of the type's lowest value
// alone; by the definition, element by element
template <typename T, int ROWT, typename SH>
__device__ Stat careful(const Row<T>& row, float scale, SH& sh) {
  const int tid = threadIdx.x % ROWT, lane = tid & 31, warp = tid / 32;
  Stat s;
  s.m = -CUDART_INF_F;
  for (int e = tid; e < row.V; e += ROWT) s.m = fmaxf(s.m, to_f32(row.x[e]));
  for (int x = 16; x; x >>= 1) s.m = fmaxf(s.m, __shfl_xor_sync(0xffffffffu, s.m, x));
  if (ROWT > 32) {
    __syncthreads();
    if (lane == 0) sh.warp[0][warp].m = s.m;
    __syncthreads();
    for (int w = 0; w < ROWT / 32; ++w) s.m = fmaxf(s.m, sh.warp[0][w].m);
  }
  s.S = s.T = 0.0f;
  if (s.m != -CUDART_INF_F)
    for (int e = tid; e < row.V; e += ROWT) {
      const float d = to_f32(row.x[e]) - s.m, p = exp_fast(d * scale);
      s.S += p;
      s.T += p == 0.0f ? 0.0f : p * d;
    }
  for (int x = 16; x; x >>= 1) {
    s.S += __shfl_xor_sync(0xffffffffu, s.S, x);
    s.T += __shfl_xor_sync(0xffffffffu, s.T, x);
  }
  if (ROWT > 32) {
    if (lane == 0) sh.warp[1][warp] = s;
    __syncthreads();
    s.S = s.T = 0.0f;
    for (int w = 0; w < ROWT / 32; ++w) {
      s.S += sh.warp[1][w].S;
      s.T += sh.warp[1][w].T;
    }
    __syncthreads();
  }
  return s;
}

// ROWT threads go through rows; with `ranks` above 1 a cluster's CTAs take one
// row's slices and the grid has a cluster for each row.
template <typename T, int ROWT> struct RowThreads {
  static constexpr int kCta = ROWT == 32 ? 128 : ROWT;
  static constexpr bool kLoop = ROWT == 32;
};

template <typename T, int ROWT, bool TOP>
__global__ void __launch_bounds__(RowThreads<T, ROWT>::kCta, (ROWT > 32 ? 1536 : TOP ? 1024 : 1280) / RowThreads<T, ROWT>::kCta) token_logp_kernel(LogpArgs a, int ranks) {
  // the next row's first loads before this one's joining: its registers would
  // cost the wide rows' CTAs a third of their warps
  constexpr bool kLoop = RowThreads<T, ROWT>::kLoop, kAhead = kLoop && !TOP;
  constexpr int U = 4, kWarps = ROWT / 32, kRows = RowThreads<T, ROWT>::kCta / ROWT;
  using C = Chunk<T>;
  __shared__ RowShared<ROWT, TOP> shared[kRows];
  RowShared<ROWT, TOP>& sh = shared[threadIdx.x / ROWT];
  const int tid = threadIdx.x % ROWT, lane = tid & 31, warp = tid / 32;
  const int rank = ranks > 1 ? blockIdx.x % ranks : 0;
  int64_t r = ranks > 1 ? blockIdx.x / ranks : (int64_t)blockIdx.x * kRows + threadIdx.x / ROWT;
  const int64_t step = ranks > 1 ? a.n : (int64_t)gridDim.x * kRows;
  pdl_enter();
  if (r >= a.n) return;  // a row's threads all leave

  uint4 v[U];
  auto slice = [&](const Row<T>& row, int& j0, int& j1) {
    const int all = row.chunks();
    j0 = ranks > 1 ? (int)((int64_t)all * rank / ranks) : 0;
    j1 = ranks > 1 ? (int)((int64_t)all * (rank + 1) / ranks) : all;
  };
  auto fetch = [&](const Row<T>& row, int64_t j, int j1) {
    if (j >= row.first_whole() && j + U * ROWT <= min(j1, row.end_whole())) {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = row.whole((int)j + u * ROWT + tid);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t jj = j + u * ROWT + tid;
        v[u] = jj < j1 ? row.any((int)jj) : make_uint4(C::kNone, C::kNone, C::kNone, C::kNone);
      }
    }
  };
  Row<T> row((const T*)a.logits + r * a.row_stride, a.V);
  int j0, j1;
  slice(row, j0, j1);
  fetch(row, j0, j1);
  for (int turn = 0;; turn ^= 1) {
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
    for (int64_t j = j0;;) {
      absorb<T, U>(v, a.scale, s);
      j += U * ROWT;
      if (j >= j1) break;
      fetch(row, j, j1);
    }
    const float mine = s.m;
    const Row<T> done = row;
    const int64_t rd = r;
    const int d0 = j0, d1 = j1;
    r += step;
    auto next = [&]() {
      row = Row<T>((const T*)a.logits + r * a.row_stride, a.V);
      slice(row, j0, j1);
      fetch(row, j0, j1);
    };
    if (kAhead && r < a.n) next();

    join_lanes<32>(s, a.scale);
    if (kWarps > 1) {
      if (lane == 0) sh.warp[turn][warp] = s;
      __syncthreads();
      s = sh.warp[turn][lane % kWarps];
      join_lanes<kWarps>(s, a.scale);
    }
    Key top = 0;
    if constexpr (TOP) top_slice<T, ROWT>(done, d0, d1, mine, a.top_k, sh);
    if (ranks > 1) {
      cg::cluster_group cl = cg::this_cluster();
      if (tid == 0) sh.slice = s;
      cl.sync();
      if (rank == 0) {
        if (lane < ranks) s = *cl.map_shared_rank(&sh.slice, lane);
        if (lane >= ranks) s = Stat{__uint_as_float(kLowBits), 0.0f, 0.0f};
        join_lanes<32>(s, a.scale);
        if (TOP && warp == 0) {
          top = sh.top[lane];
          for (int p = 1; p < ranks; ++p) top = merge_desc(top, cl.map_shared_rank(sh.top, p)[lane]);
        }
      }
      cl.sync();  // the others' shared memory has been read
      if (rank) return;
    } else if (TOP) {
      sync_row<ROWT>();
      if (warp == 0) top = sh.top[lane];
    }

    if (s.m <= __uint_as_float(kLowBits)) s = careful<T, ROWT>(done, a.scale, sh);
    const bool empty = s.m == -CUDART_INF_F;
    const float ln = logf(s.S);
    if (tid == 0) {
      if (a.lse) a.lse[rd] = empty ? -CUDART_INF_F : fmaf(s.m, a.scale, ln);
      if (a.entropy) a.entropy[rd] = empty ? 0.0f : ln - a.scale * s.T / s.S;
      if (a.logp) a.logp[rd] = t < 0 || t >= a.V ? 0.0f : empty ? -CUDART_INF_F : (zt - s.m) * a.scale - ln;
    }
    if (TOP && tid < a.top_k) {
      a.top_id[rd * a.top_k + tid] = (int32_t)(0xffffffffu - (uint32_t)top);
      a.top_logp[rd * a.top_k + tid] = empty ? -CUDART_INF_F : (key_logit((uint32_t)(top >> 32)) - s.m) * a.scale - ln;
    }
    if (!kLoop || r >= a.n) return;
    if (TOP) sync_row<ROWT>();  // the next row's candidates go where this one's were
    if (!kAhead) next();
  }
}

// ---------------------------------------------------------------------------
// gradient: THREADS threads take kGradChunks chunks each of one row; a warp a
// row where the row is short, eight of them in a CTA
// ---------------------------------------------------------------------------
constexpr int kGradChunks = 4;

template <typename T, int THREADS>
__global__ void __launch_bounds__(256) token_logp_grad_kernel(LogpGradArgs a) {
  using C = Chunk<T>;
  const int64_t r = (blockIdx.y + (int64_t)blockIdx.z * gridDim.y) * (256 / THREADS) + threadIdx.x / THREADS;
  pdl_enter();
  if (r >= a.n) return;
  const Row<T> row((const T*)a.logits + r * a.row_stride, a.V);
  T* y = (T*)a.dlogits + r * a.d_row_stride;
  const int64_t j = (int64_t)blockIdx.x * (kGradChunks * THREADS) + threadIdx.x % THREADS;
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
  const bool empty = lse == -CUDART_INF_F;  // no distribution: all zeros
  const float g = t >= 0 && t < a.V && !empty ? a.g_logp[r] : 0.0f;
  const float ge = a.g_entropy && !empty ? a.g_entropy[r] : 0.0f, H = a.g_entropy ? a.entropy[r] : 0.0f;
  // dz = p (A + B ln p)
  const float A = empty ? 0.0f : -a.scale * fmaf(ge, H, g), B = empty ? 0.0f : -a.scale * ge;
  const bool same = ((reinterpret_cast<uintptr_t>(row.x) ^ reinterpret_cast<uintptr_t>(y)) & 15) == 0;
  const float2 sc = both2(a.scale), L = both2(empty ? 0.0f : -lse), l2 = both2(kLog2e), A2 = both2(A), B2 = both2(B);
  auto gradient = [&](float2 x) {
    float2 d = __ffma2_rn(x, sc, L);
    // ln p of a forbidden token, kept finite: p is 0 there.  NaN stays
    d = make_float2(max_nan(d.x, -1000.0f), max_nan(d.y, -1000.0f));
    const float2 e = __fmul2_rn(d, l2);
    float2 p;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(p.x) : "f"(e.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(p.y) : "f"(e.y));
    return __fmul2_rn(p, __ffma2_rn(B2, d, A2));
  };
#pragma unroll
  for (int u = 0; u < kGradChunks; ++u) {
    const int64_t c = j + u * THREADS;
    if (c >= all) break;
    const bool whole = c >= w0 && c < w1;
    const uint4 in = whole ? v[u] : row.any((int)c);
    uint4 out;
#pragma unroll
    for (int i = 0; i < C::kPairs; ++i) C::put(out, i, gradient(C::pair(in, i)));
    const int place = t - (int)(c * C::kElems - row.mis);  // of the target in the chunk, which adds its own term
    if (place >= 0 && place < C::kElems)
#pragma unroll
      for (int i = 0; i < C::kPairs; ++i)
        if (i == place >> 1) {
          float2 z = gradient(C::pair(in, i));
          if (place & 1)
            z.y = fmaf(a.scale, g, z.y);
          else
            z.x = fmaf(a.scale, g, z.x);
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

template <typename T, int ROWT>
static pe_status go_logp(const LogpArgs& a, int ranks, cudaStream_t st) {
  auto kern = a.top_k ? token_logp_kernel<T, ROWT, true> : token_logp_kernel<T, ROWT, false>;
  constexpr int kCta = RowThreads<T, ROWT>::kCta, kRows = kCta / ROWT;
  cudaLaunchAttribute at[2] = {};
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = ranks;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t lc{};
  const int64_t ctas = (a.n + kRows - 1) / kRows, most = 152 * (1536 / kCta);  // what fits the SMs at 40 registers
  lc.gridDim = dim3((unsigned)(!RowThreads<T, ROWT>::kLoop ? a.n * ranks : ctas < most ? ctas : most));
  lc.blockDim = kCta;
  lc.stream = st;
  lc.attrs = at;
  lc.numAttrs = ranks > 1 ? 2 : 1;
  PE_TRY_CUDA(cudaLaunchKernelEx(&lc, kern, a, ranks));
  return PE_OK;
}

template <typename T>
static pe_status logp(const LogpArgs& a, cudaStream_t st) {
  const int64_t chunks = ceil_div(a.V, Chunk<T>::kElems);
  // Threads of a row.  Few rows, up to one 512-thread CTA in each place of the
  // SMs: eight chunks a thread, for the row's latency (one row of V = 4,096 in
  // bf16: 2.4 us with 128 threads, 4.6 with a warp).  More: sixteen, for fewer
  // partial sums a byte (8,000 rows: V = 2,000 9.9 us with a warp, 16.2 with 128;
  // V = 16,000 44 us with 128, 50 with 256).
  const bool few = a.n <= 3 * 152;
  if (chunks <= (few ? 32 : 256)) return go_logp<T, 32>(a, 1, st);
  if (chunks <= (few ? 1024 : 2048)) return go_logp<T, 128>(a, 1, st);
  // Longer rows of 256 threads where all rows fit the SMs at once (six CTAs each)
  // or fill them several times; in between 512, whose last round is shorter.
  if (chunks <= (few ? 2048 : 8192) || (!few && a.n <= 6 * 152) || a.n >= 4 * 6 * 152) return go_logp<T, 256>(a, 1, st);
  // Few rows: a cluster shares one, while each thread has four chunks and the
  // CTAs one SM each (V = 131,072 in bf16, twenty alternatives, in 1, 2, 4 and 8
  // ranks: one row 11.2, 8.7, 7.1, 7.1 us; 20 rows 13.2, 9.6, 7.9, 9.8; 64 rows
  // 13.4, 10.3, 13.8, 13.8).
  int ranks = 1;
  while (ranks < 8 && a.n * ranks * 2 <= 152 && chunks >= 512 * 4 * ranks * 2) ranks *= 2;
  return go_logp<T, 512>(a, ranks, st);
}

template <typename T, int THREADS>
static pe_status go_grad(const LogpGradArgs& a, int64_t chunks, cudaStream_t st) {
  PE_TRY_CUDA(launch_pdl(token_logp_grad_kernel<T, THREADS>, row_grid(ceil_div(chunks, kGradChunks * THREADS), ceil_div(a.n, 256 / THREADS)),
                         dim3(256), 0, st, true, a));
  return PE_OK;
}

template <typename T>
static pe_status grad(const LogpGradArgs& a, cudaStream_t st) {
  // one more where rows do not start on 16 bytes
  const bool aligned = reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 && (a.n == 1 || a.row_stride % Chunk<T>::kElems == 0);
  const int64_t chunks = (int64_t)ceil_div(a.V, Chunk<T>::kElems) + (aligned ? 0 : 1);
  return chunks <= 4 * 32 ? go_grad<T, 32>(a, chunks, st) : go_grad<T, 256>(a, chunks, st);
}

pe_status token_logp_launch(const LogpArgs& a, int dtype, cudaStream_t st) {
  ProfScope ps(PE_PROF_TOKEN_LOGP, st);
  if (dtype == PE_F32) return logp<float>(a, st);
  if (dtype == PE_BF16) return logp<__nv_bfloat16>(a, st);
  return logp<__half>(a, st);
}

pe_status token_logp_grad_launch(const LogpGradArgs& a, int dtype, cudaStream_t st) {
  ProfScope ps(PE_PROF_TOKEN_LOGP_GRAD, st);
  if (dtype == PE_F32) return grad<float>(a, st);
  if (dtype == PE_BF16) return grad<__nv_bfloat16>(a, st);
  return grad<__half>(a, st);
}

}  // namespace pe
