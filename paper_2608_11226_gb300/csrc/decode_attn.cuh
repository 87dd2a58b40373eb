// Attention of one new token per sequence over a paged cache (formulas:
// pe.h).  HBM-bound up to 16 query heads a key head: every attended key and
// value is read once, at 83% (head_dim 64) to 97% of the copy rate on long caches
// (one sequence of 262,143 positions: 162 us, 6.6 TB/s).  Beyond that a team's
// warps set the pace: each reads the whole unit from shared memory and runs a
// chain of products, softmax and shuffles of its own: 20 heads 61-76%, 32 heads
// 51-66%, 64 heads 34-41%.
//
// Work is cut into units of 16 (head_dim 64: 32) positions.  A team of HT warps
// takes a unit at a time through its own ring of cp.async stages, and a CTA's
// teams take neighbouring units, one tile.  The tiles of all (sequence, key
// head, head group) segments form one line that is dealt out evenly to the
// CTAs, so ragged lengths balance and a long cache is split without a plan on
// the host (lengths are read on the device).  At a segment's end the CTA's teams
// join in shared memory; a segment that crosses CTAs goes to the workspace as
// pieces (maxima, sums, unnormalised output), which a second kernel joins in the
// order of the CTAs.  Small batches take one cluster of CTAs per segment
// instead, joined through shared memory in the same launch.
//
// Products on mma.sync, transposed: scores S^T[16 positions x 8 heads] =
// K Q^T and O^T[D x 8 heads] += V^T P^T, so that 8 query heads fill a tile's
// columns.  tcgen05 could take the same form (positions, then head elements, as
// its rows, heads as columns); up to 16 heads a key head it has nothing to give,
// for the tensor pipe is 14% busy at the copy rate.  P enters the second product
// as a sum of two 16-bit numbers, hi + lo, which leaves 2^-18 (bf16) of a weight:
// one alone would add an error of the size of the result's own rounding.  In
// bf16 about 2 of 1,000 outputs come out a step from where fp32 weights put them,
// those whose exact value is within 1e-5 of the outputs' size of the boundary.
//
// Over 8-bit codes the same kernel runs with products in fp16, in which every code
// is exact, and units of 32 positions: fragments are loaded as pairs of codes and
// widened in registers.  A row's key scale multiplies its scores; the exponent of
// its value scale is added to them, so that the running maximum is that of weight
// times scale and P stays in fp16's range (the sum of the weights takes the scale
// out again).  Queries become fp16 with a power of two for each head.  One sequence
// of 262,143 positions, 4 heads a key head, 89 us (90% of the copy rate); 128 x up to
// 8,192, 8 heads a key head, 174 us (75%), where widening, half of the work for each
// byte, is what takes the time.
//
// Drafted nodes with few rows a key head (few_rows.cu) go through as if they were
// heads; positions that rows attend to differently, the nodes themselves and the
// first 64 of a window, are masked row by row in a path of their own.
#pragma once

#include <cooperative_groups.h>
#include <math_constants.h>

#include <cmath>
#include <type_traits>

#include "tokens.cuh"

namespace pe {

namespace cg = cooperative_groups;

constexpr int kMaxRanks = 8;          // CTAs of a cluster
constexpr int kDecodeCtas = 152 * 2;  // CTAs of the line at most: two on each SM

template <typename T> struct Mma;
template <> struct Mma<__nv_bfloat16> {
  static constexpr float kBias = 0.0f;
  static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};
template <> struct Mma<__half> {
  // weights are e^(s - m) 2^6, at most 2^14: fp16 keeps what is 2^-30 of the
  // largest, so a long tail of small weights is not lost
  static constexpr float kBias = 6.0f;
  static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};

// type of the products
template <typename T, bool E8> using Product = typename std::conditional<E8, __half, T>::type;

// codes 2 i and 2 i + 1 of a word, widened
__device__ __forceinline__ uint32_t widen(uint32_t w, int i) {
  uint32_t v;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(v) : "h"((uint16_t)(w >> (16 * i))));
  return v;
}

__device__ __forceinline__ void ldsm(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
// 16 bytes into shared memory, zeros where !ok (the address is not read then)
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
// 2^x within 2^-22, far below what hi + lo leave of a weight
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// hi and lo parts of two weights, packed
template <typename T>
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo) {
  hi = pack2<T>(a, b);
  const float2 h = unpack2<T>(hi);
  lo = pack2<T>(a - h.x, b - h.y);
}

// a segment that crosses CTAs, as the joining kernel finds it: pieces in slot
// first_slot, then in the first slots of the CTAs after it
struct SegMeta {
  int32_t seq, head_group, pieces, first_slot;  // pieces 0: nothing to join
};

// E8: 8-bit codes
template <bool E8, int D, int NT, int HT>
struct DecodeShape {
  // wide heads leave one CTA on an SM: more warps where its teams have several
  static constexpr int kWarps = D == 256 && HT > 1 ? (HT == 3 ? 12 : 8) : 4;
  static constexpr int kThreads = 32 * kWarps;
  static constexpr int kTeams = kWarps / HT;
  static constexpr int kBlocks = D == 256 ? 1 : 2;  // CTAs on an SM
  static constexpr int kCtas = 152 * kBlocks;
  static constexpr int kHeads = 8 * NT * HT;            // query heads of a segment
  static constexpr int kUnit = E8 || D == 64 || (D == 128 && HT > 1) || (D == 256 && HT == 4) ? 32 : 16;  // positions of a stage
  static constexpr int kRowBytes = E8 ? D : 2 * D;
  static constexpr int kUnitBytes = 2 * kUnit * kRowBytes;  // its keys and values
  // a ring of 96 KB (two CTAs on an SM) or, for wide heads, 192 KB; at most 8 stages
  static constexpr int kFit = (kBlocks == 1 ? 196608 : 98304) / (kTeams * kUnitBytes);
  static constexpr int kStages = kFit > (E8 ? 4 : 8) ? (E8 ? 4 : 8) : kFit;
  static constexpr int kRing = kTeams * kStages * kUnitBytes;
  static constexpr int kPiece = 8 * NT * (D + 2);       // floats of a warp's piece: output, maxima, sums
  static constexpr int kTiles = NT * (D / 16);          // 16 x 8 tiles of its output
  // the teams join `kRound` tiles of each warp at a time
  static constexpr int kAtOnce = E8 || NT > 2 || kWarps > 4 ? 4 : 8;
  static constexpr int kRound = kTeams == 1 ? 0 : kAtOnce < kTiles ? kAtOnce : kTiles;
  static constexpr int kMerge = kWarps * (kRound * 512 + 2 * 8 * NT * 4);
  static constexpr int kWeights = kMaxRanks * kTeams * kHeads * 8;
  static constexpr int kExtra = kMerge > kWeights ? kMerge : kWeights;
  static constexpr int kSmem = kRing + kExtra;  // prefix sums at first, then what joins the teams, or the cluster
  static_assert(HT * kPiece * 4 <= kStages * kUnitBytes, "a team's piece in place of its ring");
  static_assert(!E8 || kStages >= 3, "a unit's scales are written a unit before it is read");
  static constexpr int kScales = E8 ? kTeams * kStages * kUnit * 16 : 0;  // static shared memory
  static_assert(kBlocks == 1 ? kSmem + kScales <= 231000 : 2 * (kSmem + kScales + 1024 + 512) <= 233472, "shared memory of an SM");
};

struct Segment {
  int b, h, hk;     // sequence, head group, key head
  int nt;           // tiles
  int base, lo, n;  // position of the first (a multiple of the unit), attended range [lo, n)
  int ctx;          // of drafted nodes: where they start
  int ahead;        // length of the next sequence, on its way
};

// nt counts tiles of `tile` positions; base is a multiple of `align`
template <bool TREE>
__device__ __forceinline__ void seq_range(const DecodeArgs& a, int len, int align, int tile, Segment& s) {
  const int cap = a.c.max_pages * a.c.page_size;
  s.n = min(max(len, 0), cap);
  s.lo = a.window > 0 ? max(0, s.n + (TREE ? 1 : 0) - a.window) : 0;
  if (TREE) s.ctx = s.n, s.n = min(cap, s.n + a.n_nodes);
  s.base = s.lo & ~(align - 1);
  s.nt = max(1, (s.n - s.base + tile - 1) / tile);  // an empty sequence has one empty tile
}
template <bool TREE>
__device__ __forceinline__ void next_segment(const DecodeArgs& a, int groups, int per_head, int align, int tile, Segment& s) {
  if (++s.h < groups) {
    s.hk = s.h / per_head;
    return;
  }
  s.h = s.hk = 0;
  ++s.b;
  seq_range<TREE>(a, s.ahead, align, tile, s);
  s.ahead = a.lens[min(s.b + 1, a.c.n_seqs - 1)];
}

// the weight of a piece with maximum m where the largest is mm; a piece that
// met nothing has m = -inf, sum 0 and output 0
__device__ __forceinline__ float piece_weight(float m, float mm) {
  return m == -CUDART_INF_F ? (mm == -CUDART_INF_F ? 1.0f : 0.0f) : exp2_fast(m - mm);
}
template <typename T> __device__ __forceinline__ float log_sum(float mm, float sum) {
  return sum == 0.0f ? -CUDART_INF_F : (mm == -CUDART_INF_F ? 0.0f : mm - Mma<T>::kBias) * 0.69314718f + logf(sum);
}

// One 16 x 8 tile of O^T (rows kk * 16 on, heads `head` on) as the product
// leaves it in a warp, scaled by the lane's two heads' factors: transposed in
// registers, so that a lane writes two neighbouring elements of one head.
// Over codes the rows of a tile are the elements 0, 2, ... 14, 1, 3, ... 15.
// `out` is the row of head lane / 4.
template <typename T, bool E8>
__device__ __forceinline__ void store_tile(T* out, int heads, int kk, float4 o, float f0, float f1) {
  const int lane = threadIdx.x & 31;
  // a factor of 0 stands for a sum of 0, nothing attended to
  const uint32_t lo = transpose8(pack2<T>(f0 == 0.0f ? 0.0f : o.x * f0, f1 == 0.0f ? 0.0f : o.y * f1));
  const uint32_t hi = transpose8(pack2<T>(f0 == 0.0f ? 0.0f : o.z * f0, f1 == 0.0f ? 0.0f : o.w * f1));
  if (lane / 4 < heads) {
    if constexpr (E8) {
      *reinterpret_cast<uint2*>(out + kk * 16 + 4 * (lane & 3)) =
          make_uint2(__byte_perm(lo, hi, 0x5410), __byte_perm(lo, hi, 0x7632));
    } else {
      uint32_t* p = reinterpret_cast<uint32_t*>(out + kk * 16 + 2 * (lane & 3));
      p[0] = lo;
      p[4] = hi;
    }
  }
}

// A lane's part of a tile, joined over pieces: unnormalised output of its two
// heads, their maxima and sums.
struct Joined {
  float4 x;
  float2 m, l;
  __device__ __forceinline__ Joined() : x(make_float4(0.0f, 0.0f, 0.0f, 0.0f)), m(make_float2(-HUGE_VALF, -HUGE_VALF)), l(make_float2(0.0f, 0.0f)) {}
  __device__ __forceinline__ void rescale(float2 top) {
    const float2 f = make_float2(piece_weight(m.x, top.x), piece_weight(m.y, top.y));
    m = top;
    l = make_float2(l.x * f.x, l.y * f.y);
    x = make_float4(x.x * f.x, x.y * f.y, x.z * f.x, x.w * f.y);
  }
  __device__ __forceinline__ void add(float2 pm, float2 pl, float4 v) {  // a piece whose maxima are at most m
    const float2 f = make_float2(piece_weight(pm.x, m.x), piece_weight(pm.y, m.y));
    l = make_float2(fmaf(f.x, pl.x, l.x), fmaf(f.y, pl.y, l.y));
    x = make_float4(fmaf(f.x, v.x, x.x), fmaf(f.y, v.y, x.y), fmaf(f.x, v.z, x.z), fmaf(f.y, v.w, x.w));
  }
  // pieces i0, i0 + step, ... below n, `kBatch` in flight at a time; `at(i)`: piece i of the warp, whose `heads`
  // heads' output comes first, then maxima, then sums
  template <int kBatch, typename F>
  __device__ __forceinline__ void gather(int i0, int step, int n, F at, int64_t x_at, int64_t m_at, int heads) {
    for (; i0 < n; i0 += kBatch * step) {
      float4 v[kBatch];
      float2 pm[kBatch], pl[kBatch], top = m;
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int i = i0 + u * step;
        pm[u] = make_float2(-CUDART_INF_F, -CUDART_INF_F);
        pl[u] = make_float2(0.0f, 0.0f);
        v[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (i >= n) continue;
        const float* p = at(i);
        pm[u] = *reinterpret_cast<const float2*>(p + m_at);
        pl[u] = *reinterpret_cast<const float2*>(p + m_at + heads);
        v[u] = *reinterpret_cast<const float4*>(p + x_at);
      }
#pragma unroll
      for (int u = 0; u < kBatch; ++u) top = make_float2(fmaxf(top.x, pm[u].x), fmaxf(top.y, pm[u].y));
      rescale(top);
#pragma unroll
      for (int u = 0; u < kBatch; ++u) add(pm[u], pl[u], v[u]);
    }
  }
};

// The line of `total` tiles dealt out to `workers` CTAs: the first `more` get one
// more than the others.
struct Deal {
  int64_t each;
  int more;
  __device__ __forceinline__ Deal(int64_t total, int workers) {
    each = total >> 32 ? total / workers : (int64_t)((uint32_t)total / (uint32_t)workers);
    more = (int)(total - each * workers);
  }
  __device__ __forceinline__ int64_t start(int w) const { return w * each + min(w, more); }
  __device__ __forceinline__ int worker(int64_t tile) const {
    const int64_t cut = more * (each + 1);
    return tile < cut ? (int)(tile / (each + 1)) : more + (int)((tile - cut) / each);
  }
};

// Rows of a key head: its g query heads, for drafted nodes (TREE) those of every
// node, one node after the other.
template <bool TREE> __device__ __forceinline__ int rows_of(const DecodeArgs& a, int g) { return g * (TREE ? a.n_nodes : 1); }
// offset of row r within a sequence's queries or output
template <bool TREE>
__device__ __forceinline__ int64_t row_at(int g, int hk, int r, int64_t node_stride, int64_t head_stride) {
  if (!TREE) return ((int64_t)hk * g + r) * head_stride;
  const int node = r / g;
  return node * node_stride + ((int64_t)hk * g + r - node * g) * head_stride;
}
template <bool TREE> __device__ __forceinline__ int64_t lse_at(const DecodeArgs& a, int seq, int g, int hk, int r) {
  if (!TREE) return (int64_t)seq * a.n_q_heads + (int64_t)hk * g + r;
  const int node = r / g;
  return ((int64_t)seq * a.n_nodes + node) * a.n_q_heads + (int64_t)hk * g + r - node * g;
}
// mask of a row's node; 0 where there is none
__device__ __forceinline__ uint64_t node_bits(const DecodeArgs& a, int seq, int r) {
  const int node = r / (a.n_q_heads / a.c.n_heads);
  return node < a.n_nodes ? a.mask[seq * a.mask_stride + node] & (0xffffffffffffffffull >> (64 - a.n_nodes)) : 0;
}

// the result of a tile: eight rows from `r` on, of which `rows` exist
template <typename T, bool E8, bool TREE>
__device__ __forceinline__ void finish(const DecodeArgs& a, int seq, int g, int hk, int r, int rows, int kk, const Joined& j) {
  const int lane = threadIdx.x & 31;
  if (kk == 0 && lane < 4 && a.lse) {
    if (2 * lane < rows) a.lse[lse_at<TREE>(a, seq, g, hk, r + 2 * lane)] = log_sum<Product<T, E8>>(j.m.x, j.l.x);
    if (2 * lane + 1 < rows) a.lse[lse_at<TREE>(a, seq, g, hk, r + 2 * lane + 1)] = log_sum<Product<T, E8>>(j.m.y, j.l.y);
  }
  store_tile<T, E8>((T*)a.out + seq * a.o_seq + row_at<TREE>(g, hk, r + lane / 4, a.o_node, a.o_head), rows, kk, j.x,
                    j.l.x == 0.0f ? 0.0f : 1.0f / j.l.x, j.l.y == 0.0f ? 0.0f : 1.0f / j.l.y);
}

// CL: one cluster for each segment, whose teams share its units and join in
// shared memory; otherwise the line of all tiles, dealt out to the CTAs, at
// least `least` to each.  by_seg: the joining kernel goes by segments and not
// by CTAs.  TREE: drafted nodes.
template <typename T, bool E8, int D, int NT, int HT, bool CL, bool TREE>
__global__ void __launch_bounds__(DecodeShape<E8, D, NT, HT>::kThreads, DecodeShape<E8, D, NT, HT>::kBlocks)
    decode_attn_kernel(DecodeArgs a, int groups, int per_head, int page_shift, int ranks, int least, bool by_seg, float* part, SegMeta* meta) {
  using S = DecodeShape<E8, D, NT, HT>;
  using W = Product<T, E8>;
  using M = Mma<W>;
  using E = typename std::conditional<E8, uint8_t, T>::type;  // element of the cache
  constexpr int kRow = S::kRowBytes, kChunks = kRow / 16, kPer = 16 / sizeof(E);
  constexpr int kTeams = S::kTeams, kStages = S::kStages, kUnit = S::kUnit;
  constexpr uint32_t kAll = 0xffffffffu >> (32 - kUnit);
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int s_where[4];
  __shared__ uint32_t s_mask[kTeams][kStages];
  // of each position: key scale, exponent of the value scale, and 2 to minus that
  __shared__ float4 s_scale[E8 ? kTeams : 1][E8 ? kStages : 1][E8 ? kUnit : 1];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int team = warp / HT, hw = warp % HT;
  const pe_kv_cache& c = a.c;
  const int B = c.n_seqs;
  // a CTA's teams take a tile's units, or a team of a cluster its own range of them
  constexpr int kTile = CL ? kUnit : kTeams * kUnit;

  int64_t start, end;  // tiles of the line, or of the segment
  int first;           // tile of the segment that start is
  Deal deal(1, 1);
  Segment cs;          // the segment computed on
  cudaGridDependencySynchronize();
  cudaTriggerProgrammaticLaunchCompletion();
  if constexpr (CL) {
    const int seg = blockIdx.x / ranks, worker = blockIdx.x % ranks * kTeams + team;
    cs.b = seg / groups;
    cs.h = seg % groups;
    seq_range<TREE>(a, a.lens[cs.b], kUnit, kTile, cs);
    start = (int64_t)cs.nt * worker / (ranks * kTeams);
    end = (int64_t)cs.nt * (worker + 1) / (ranks * kTeams);
    first = (int)start;
  } else {
    // a prefix sum of the sequences' tiles finds where this CTA's share starts
    int64_t* s_sum = reinterpret_cast<int64_t*>(smem + S::kRing);
    const int chunk = (B + S::kThreads - 1) / S::kThreads;
    int64_t sum = 0;
    int len = 0;
    Segment s;
    for (int b = tid * chunk; b < min(B, (tid + 1) * chunk); ++b) {
      len = a.lens[b];
      seq_range<TREE>(a, len, kUnit, kTile, s);
      sum += s.nt;
    }
    int64_t incl = sum;
    for (int x = 1; x < 32; x <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, incl, x);
      if (lane >= x) incl += y;
    }
    if (lane == 31) s_sum[warp] = incl;
    __syncthreads();
    int64_t before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < S::kWarps; ++w) {
      const int64_t x = s_sum[w];
      if (w < warp) before += x;
      total += x;
    }
    total *= groups;
    const int64_t most = (total + least - 1) / least;
    const int workers = most < gridDim.x ? (int)most : (int)gridDim.x;
    if (blockIdx.x >= workers) {
      if (!by_seg && tid == 0) meta[blockIdx.x].pieces = 0;
      return;
    }
    deal = Deal(total, workers);
    start = deal.start(blockIdx.x);
    end = deal.start(blockIdx.x + 1);
    const int64_t lo = (before + incl - sum) * groups, hi = (before + incl) * groups;
    if (start >= lo && start < hi) {
      int64_t at = lo;
      int b = tid * chunk;
      if (chunk > 1)
        for (;; ++b) {
          len = a.lens[b];
          seq_range<TREE>(a, len, kUnit, kTile, s);
          if (start < at + (int64_t)s.nt * groups) break;
          at += (int64_t)s.nt * groups;
        }
      const int64_t in = start - at;
      const int h = in >> 32 ? (int)(in / s.nt) : (int)((uint32_t)in / (uint32_t)s.nt);
      s_where[0] = b;
      s_where[1] = h;
      s_where[2] = (int)(in - (int64_t)h * s.nt);
      s_where[3] = len;
    }
    __syncthreads();
    cs.b = s_where[0];
    cs.h = s_where[1];
    first = s_where[2];
    seq_range<TREE>(a, s_where[3], kUnit, kTile, cs);
    if (!by_seg && tid == 0) {
      // the boundary at this CTA's start joins the segment if it is the first inside it
      const int64_t g0 = start - first, prev = deal.start((int)blockIdx.x - 1);
      SegMeta m{cs.b, cs.h, 0, 0};
      if (first > 0 && prev <= g0) {
        m.pieces = deal.worker(g0 + cs.nt - 1) - blockIdx.x + 2;
        m.first_slot = 2 * (blockIdx.x - 1) + (prev < g0 ? 1 : 0);
      }
      meta[blockIdx.x] = m;
    }
  }
  cs.hk = cs.h / per_head;
  cs.ahead = a.lens[min(cs.b + 1, B - 1)];

  // -- loading: kStages - 1 units ahead of the computation; a unit's page is
  // looked up one unit before that
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + team * kStages * S::kUnitBytes;
  const int at0 = CL ? 0 : team * kUnit;                // place of the team's unit in a tile
  const bool one_page = c.page_size % kUnit == 0;  // no unit crosses a page
  const bool two_pages = E8 && c.page_size % 16 == 0;  // no half of one does
  // place of a 16-byte chunk in its row, so that ldmatrix' eight rows meet no bank twice
  auto swizzle = [](int row, int ch) { return E8 && D == 64 ? ch ^ ((row >> 1) & 3) : ch ^ (row & 7); };
  Segment ls = cs;
  int kbyte = 0, vbyte = 0, scale_stage = -1;  // scales on their way
  auto store_scales = [&]() {  // of the unit loaded before
    if (E8 && scale_stage >= 0 && hw == 0) {
      const int e = min(max(vbyte, 63), 247);
      s_scale[team][scale_stage][lane] =
          kbyte < 0 ? make_float4(0.0f, 0.0f, 1.0f, 0.0f)
                    : make_float4(key_scale(kbyte), vbyte == 255 ? CUDART_NAN_F : (float)(e - 127), __int_as_float((254 - e) << 23), 0.0f);
    }
    scale_stage = -1;
  };
  int lt = first, lstage = 0, lslot, lpage;
  int lleft = (int)(end - start);
  auto aim = [&]() {  // the page of the next unit, or of the lane's position in it
    const int pos = ls.base + lt * kTile + at0 + (one_page ? 0 : lane & (kUnit - 1));
    const int p = page_shift >= 0 ? pos >> page_shift : pos / c.page_size;
    lslot = pos - p * c.page_size;
    lpage = one_page || pos >= ls.lo ? pos < ls.n ? c.table[(int64_t)ls.b * c.table_stride + p] : -1 : -1;
  };
  auto load = [&]() {
    if (E8) store_scales();
    if (lleft > 0) {
      constexpr int kRows = 32 / kChunks * HT;                 // rows of one copy instruction of each warp
      constexpr int kCopies = (kUnit + kRows - 1) / kRows;
      const int row0 = lane / kChunks * HT + hw, ch = lane % kChunks;
      const uint32_t dst = ring + lstage * S::kUnitBytes + row0 * kRow;
      const bool ok = lpage >= 0 && lpage < c.n_pages;
      int64_t off = ok ? kv_page_offset(c, lpage) + (int64_t)lslot * c.slot_stride + ls.hk * c.head_stride : 0;
      uint32_t mask;
      if (one_page) {
        const int at = ls.base + lt * kTile + at0;
        const int r0 = max(ls.lo - at, 0), r1 = min(ls.n - at, kUnit);  // attended rows
        mask = ok && r1 > 0 ? (kAll >> (kUnit - r1)) & (kAll << r0) : 0u;
      } else {
        mask = __ballot_sync(0xffffffffu, ok) & kAll;
      }
      if (lane == 0 && hw == 0) s_mask[team][lstage] = mask;
      if (E8) {  // a lane for each position
        scale_stage = lstage;
        kbyte = vbyte = -1;
        if (hw == 0 && ((mask >> lane) & 1)) {
          const int64_t so = (int64_t)lpage * a.sc.page_stride + (int64_t)(one_page ? lslot + lane : lslot) * a.sc.slot_stride + ls.hk * a.sc.head_stride;
          kbyte = a.sc.k[so];
          vbyte = a.sc.v[so];
        }
      }
      if (one_page && mask == kAll) {
        const E* k = (const E*)c.k + off + row0 * c.slot_stride + ch * kPer;
        const E* v = (const E*)c.v + off + row0 * c.slot_stride + ch * kPer;
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
          if (kUnit % kRows != 0 && row0 + i * kRows >= kUnit) break;
          const uint32_t d = dst + i * kRows * kRow + (swizzle(row0 + i * kRows, ch) << 4);
          copy16(d, k + i * kRows * c.slot_stride, true);
          copy16(d + kUnit * kRow, v + i * kRows * c.slot_stride, true);
        }
      } else if (two_pages && mask == kAll) {
        const E* base[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int64_t o = __shfl_sync(0xffffffffu, off, 16 * h) + (int64_t)(row0 - 16 * h) * c.slot_stride + ch * kPer;
          base[h][0] = (const E*)c.k + o;
          base[h][1] = (const E*)c.v + o;
        }
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
          const int row = row0 + i * kRows;
          if (kUnit % kRows != 0 && row >= kUnit) break;
          const bool h = 16 % kRows == 0 ? i * kRows >= 16 : row >= 16;
          const uint32_t d = dst + i * kRows * kRow + (swizzle(row, ch) << 4);
          copy16(d, (h ? base[1][0] : base[0][0]) + i * kRows * c.slot_stride, true);
          copy16(d + kUnit * kRow, (h ? base[1][1] : base[0][1]) + i * kRows * c.slot_stride, true);
        }
      } else {
        if (one_page && lane & (kUnit - 1)) off += (lane & (kUnit - 1)) * c.slot_stride;
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
          const int row = row0 + i * kRows;
          const int64_t o = __shfl_sync(0xffffffffu, off, row & 31) + ch * kPer;
          if (kUnit % kRows != 0 && row >= kUnit) continue;
          const bool in = (mask >> row) & 1;
          const uint32_t d = dst + i * kRows * kRow + (swizzle(row, ch) << 4);
          copy16(d, (const E*)c.k + (in ? o : 0), in);
          copy16(d + kUnit * kRow, (const E*)c.v + (in ? o : 0), in);
        }
      }
      --lleft;
      if (++lt == ls.nt) {
        lt = 0;
        if (!CL && lleft > 0) next_segment<TREE>(a, groups, per_head, kUnit, kTile, ls);
      }
      if (lleft > 0) aim();
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    lstage = lstage + 1 == kStages ? 0 : lstage + 1;
  };
  const int mine = (int)(end - start);
  if (lleft > 0) aim();
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) load();

  // -- computing
  // ldmatrix places of the lane: row, and 16-byte column under the ring's
  // swizzle, whose three bits repeat every 128 bytes of a row
  uint32_t kat[4], vat[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // (four matrices of 8 rows x 16 bytes; of codes both operands' are rows 0 on and 8 on, 32 elements)
    const int kr = lane & 15, vr = E8 ? kr : (lane & 7) + 8 * (lane / 16);
    kat[i] = kr * kRow + (swizzle(kr, i * 2 + lane / 16) << 4);
    vat[i] = kUnit * kRow + vr * kRow + (swizzle(vr, E8 ? i * 2 + lane / 16 : i * 2 + ((lane >> 3) & 1)) << 4);
  }
  auto team_sync = [&]() {
    if (HT == 1)
      __syncwarp();
    else
      asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(32 * HT) : "memory");
  };
  const float qscale = a.scale * 1.4426950408889634f * (E8 ? kRowFactor : 1.0f);  // scores in powers of two
  const int g = a.n_q_heads / c.n_heads, group = rows_of<TREE>(a, g);  // query heads, rows of a key head
  uint32_t qf[D / 16][NT][2];
  float o[D / 16][NT][4], m[NT][2], l[NT][2];
  float qc[E8 ? NT : 1][2];  // of the lane's heads: scale over the query's power of two
  auto load_q = [&]() {
    const T* q = (const T*)a.q + cs.b * a.q_seq;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int h = (cs.h - cs.hk * per_head) * S::kHeads + hw * 8 * NT + nt * 8 + lane / 4;
      const T* row = q + row_at<TREE>(g, cs.hk, h < group ? h : 0, a.q_node, a.q_head);
      if constexpr (E8) {
        // the elements that a lane's four codes meet, in fp16 with the row's largest in [2^14, 2^15)
        uint2 w[D / 16];
        uint32_t most = 0;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          w[kk] = h < group ? *reinterpret_cast<const uint2*>(row + kk * 16 + 4 * (lane & 3)) : make_uint2(0, 0);
          const float2 x = unpack2<T>(w[kk].x), y = unpack2<T>(w[kk].y);
          most = max(max(most, max(__float_as_uint(x.x) & 0x7fffffffu, __float_as_uint(x.y) & 0x7fffffffu)),
                     max(__float_as_uint(y.x) & 0x7fffffffu, __float_as_uint(y.y) & 0x7fffffffu));
        }
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const int ex = (int)(most >> 23);
        const int up = ex == 255 || most == 0 ? 127 : min(268 - ex, 253);  // exponent field of the factor
        const float f = __uint_as_float((uint32_t)up << 23), back = __uint_as_float((uint32_t)(254 - up) << 23);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const float2 x = unpack2<T>(w[kk].x), y = unpack2<T>(w[kk].y);
          qf[kk][nt][0] = pack2<__half>(x.x * f, x.y * f);
          qf[kk][nt][1] = pack2<__half>(y.x * f, y.y * f);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) qc[nt][i] = qscale * __shfl_sync(0xffffffffu, back, 8 * (lane & 3) + 4 * i);
      } else {
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint32_t* p = reinterpret_cast<const uint32_t*>(row + kk * 16 + 2 * (lane & 3));
          qf[kk][nt][0] = h < group ? p[0] : 0u;
          qf[kk][nt][1] = h < group ? p[4] : 0u;
        }
      }
    }
  };
  auto reset = [&]() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[kk][nt][i] = 0.0f;
      m[nt][0] = m[nt][1] = -CUDART_INF_F;
      l[nt][0] = l[nt][1] = 0.0f;
    }
  };
  auto sum_lanes = [&](int seq) {  // l over the lanes that hold a head's positions
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (TREE && node_bits(a, seq, hw * 8 * NT + nt * 8 + 2 * (lane & 3) + i) == 0) m[nt][i] = -CUDART_INF_F, l[nt][i] = 0.0f;  // padding
        l[nt][i] += __shfl_xor_sync(0xffffffffu, l[nt][i], 4);
        l[nt][i] += __shfl_xor_sync(0xffffffffu, l[nt][i], 8);
        l[nt][i] += __shfl_xor_sync(0xffffffffu, l[nt][i], 16);
      }
  };
  auto store_piece = [&](float* p) {  // as the registers hold it; then maxima and sums
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
        reinterpret_cast<float4*>(p)[(nt * (D / 16) + kk) * 32 + lane] = make_float4(o[kk][nt][0], o[kk][nt][1], o[kk][nt][2], o[kk][nt][3]);
      if (lane < 4) {
        *reinterpret_cast<float2*>(p + 8 * NT * D + nt * 8 + 2 * lane) = make_float2(m[nt][0], m[nt][1]);
        *reinterpret_cast<float2*>(p + 8 * NT * (D + 1) + nt * 8 + 2 * lane) = make_float2(l[nt][0], l[nt][1]);
      }
    }
  };
  // A unit that rows attend to differently (drafted nodes, the head of a window): scores that a row leaves out,
  // and values that are not finite, which become zero and make the elements of those who attend NaN.
  auto by_row = [&](int p0, uint32_t unit, float (&s)[kUnit / 16][NT][4]) {
    uint64_t bits[NT][2];
    int row_lo[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        bits[nt][i] = node_bits(a, cs.b, hw * 8 * NT + nt * 8 + 2 * (lane & 3) + i);
        row_lo[nt][i] = a.window > 0 ? max(0, cs.ctx + __popcll(bits[nt][i]) - a.window) : 0;
      }
    auto attends = [&](int nt, int i, int p) {
      return p < cs.ctx ? bits[nt][i] != 0 && p >= row_lo[nt][i] : p - cs.ctx < 64 && ((bits[nt][i] >> (p - cs.ctx)) & 1);
    };
#pragma unroll
    for (int u = 0; u < kUnit / 16; ++u)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!attends(nt, i & 1, p0 + 16 * u + lane / 4 + 8 * (i / 2))) s[u][nt][i] = -CUDART_INF_F;
    unsigned char* values = smem + (unit - (uint32_t)__cvta_generic_to_shared(smem)) + kUnit * kRow;
    auto none = [](uint32_t w, int i) {  // element i of a word
      return E8 ? ((w >> (8 * i)) & 0x7f) == 0x7f : ((w >> (16 * i)) & (std::is_same<T, __nv_bfloat16>::value ? 0x7f80u : 0x7c00u)) ==
                                                        (std::is_same<T, __nv_bfloat16>::value ? 0x7f80u : 0x7c00u);
    };
    constexpr int kIn = E8 ? 4 : 2;  // elements of a word
    uint32_t rows = 0;
#pragma unroll 1
    for (int x = lane; x < kUnit * kRow / 4; x += 32) {
      const uint32_t w = reinterpret_cast<const uint32_t*>(values)[x];
#pragma unroll
      for (int i = 0; i < kIn; ++i)
        if (none(w, i)) rows |= 1u << (x / (kRow / 4));
    }
    rows = __reduce_or_sync(0xffffffffu, rows);
    if (__builtin_expect(rows == 0, 1)) return;
#pragma unroll 1
    for (int r = 0; r < kUnit; ++r) {
      if (!((rows >> r) & 1)) continue;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int e = kk * 16 + (E8 ? 2 * (lane / 4) + half : lane / 4 + 8 * half), byte = e * (int)sizeof(E);
          const unsigned char* at = values + r * kRow + (swizzle(r, byte >> 4) << 4) + (byte & 15);
          if (!none(E8 ? *at : *reinterpret_cast<const uint16_t*>(at), 0)) continue;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              if (attends(nt, i, p0 + r)) o[kk][nt][2 * half + i] = CUDART_NAN_F;
        }
    }
    team_sync();  // the team's warps have all looked
#pragma unroll 1
    for (int x = lane; x < kUnit * kRow / 4; x += 32) {  // (each of them: the same words)
      uint32_t w = reinterpret_cast<const uint32_t*>(values)[x];
#pragma unroll
      for (int i = 0; i < kIn; ++i)
        if (none(w, i)) w &= ~((E8 ? 0xffu : 0xffffu) << ((E8 ? 8 : 16) * i));
      reinterpret_cast<uint32_t*>(values)[x] = w;
    }
    team_sync();
  };
  load_q();
  reset();
  int ct = first, stage = 0;
  bool from_first = first == 0;  // this CTA holds the segment's first tile
  for (int left = mine; left > 0; --left) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
    team_sync();
    load();
    const uint32_t unit = ring + stage * S::kUnitBytes;
    const uint32_t mask = s_mask[team][stage];
    const float4* scales = s_scale[E8 ? team : 0][E8 ? stage : 0];
    stage = stage + 1 == kStages ? 0 : stage + 1;
    if (mask) {
      // scores of 16 positions at a time; two chains of products where one
      // head tile gives only one
      constexpr int kSub = kUnit / 16, kChains = NT == 1 ? 2 : 1;
      float s[kSub][NT][4];
      float el[E8 ? kSub : 1][2];  // what takes a position's value scale out of a weight
#pragma unroll
      for (int u = 0; u < kSub; ++u) {
        float s2[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) s[u][nt][i] = 0.0f;
          s2[i] = 0.0f;
        }
        if constexpr (E8) {
#pragma unroll
          for (int k2 = 0; k2 < D / 32; ++k2) {
            uint32_t w[4];
            ldsm(w, unit + kat[k2 & 3] + (k2 >> 2) * 128 + u * 16 * kRow);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const uint32_t f[4] = {widen(w[2 * x], 0), widen(w[2 * x + 1], 0), widen(w[2 * x], 1), widen(w[2 * x + 1], 1)};
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) M::mma(kChains == 2 && x ? s2 : s[u][nt], f, qf[2 * k2 + x][nt][0], qf[2 * k2 + x][nt][1]);
            }
          }
          const float4 r0 = scales[16 * u + lane / 4], r1 = scales[16 * u + lane / 4 + 8];
          el[u][0] = r0.z, el[u][1] = r1.z;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (kChains == 2) s[u][0][i] += s2[i];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[u][nt][i] = fmaf(s[u][nt][i] * (i < 2 ? r0.x : r1.x), qc[nt][i & 1], i < 2 ? r0.y : r1.y);
          }
        } else {
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            uint32_t f[4];
            ldsm(f, unit + kat[kk & 3] + (kk >> 2) * 128 + u * 16 * D * 2);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) M::mma(kChains == 2 && (kk & 1) ? s2 : s[u][nt], f, qf[kk][nt][0], qf[kk][nt][1]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (kChains == 2) s[u][0][i] += s2[i];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[u][nt][i] *= qscale;
          }
        }
      }
      if (mask != kAll) {
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
          const bool r0 = (mask >> (lane / 4 + 16 * u)) & 1, r1 = (mask >> (lane / 4 + 8 + 16 * u)) & 1;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            if (!r0) s[u][nt][0] = s[u][nt][1] = -CUDART_INF_F;
            if (!r1) s[u][nt][2] = s[u][nt][3] = -CUDART_INF_F;
          }
        }
      }
      if constexpr (TREE) {
        const int p0 = cs.base + ct * kTile + at0;
        if (p0 + kUnit > cs.ctx || (a.window > 0 && p0 < cs.lo + 64)) by_row(p0, unit, s);
      }
      // the reference of the exponentials follows the maximum only when it is
      // passed by 8 (a factor of 256): few units rescale
      bool over = false;
#pragma unroll
      for (int u = 0; u < kSub; ++u)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) over |= s[u][nt][i] > m[nt][i & 1] + 8.0f;
      if (__any_sync(0xffffffffu, over)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float x = m[nt][i];
#pragma unroll
            for (int u = 0; u < kSub; ++u) x = fmaxf(x, fmaxf(s[u][nt][i], s[u][nt][i + 2]));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
            const float f = m[nt][i] == -CUDART_INF_F ? 0.0f : exp2_fast(m[nt][i] - x);
            m[nt][i] = x;
            l[nt][i] *= f;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
              o[kk][nt][i] *= f;
              o[kk][nt][i + 2] *= f;
            }
          }
      }
#pragma unroll
      for (int u = 0; u < kSub; ++u) {
        uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float r0 = (m[nt][0] == -CUDART_INF_F ? 0.0f : m[nt][0]) - M::kBias;
          const float r1 = (m[nt][1] == -CUDART_INF_F ? 0.0f : m[nt][1]) - M::kBias;
          const float p0 = exp2_fast(s[u][nt][0] - r0), p1 = exp2_fast(s[u][nt][1] - r1);
          const float p2 = exp2_fast(s[u][nt][2] - r0), p3 = exp2_fast(s[u][nt][3] - r1);
          if constexpr (E8) {
            l[nt][0] = fmaf(p0, el[u][0], fmaf(p2, el[u][1], l[nt][0]));
            l[nt][1] = fmaf(p1, el[u][0], fmaf(p3, el[u][1], l[nt][1]));
          } else {
            l[nt][0] += p0 + p2;
            l[nt][1] += p1 + p3;
          }
          split2<W>(p0, p1, ph[nt][0], pl[nt][0]);
          split2<W>(p2, p3, ph[nt][1], pl[nt][1]);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            ph[nt][i] = transpose8(ph[nt][i]);
            pl[nt][i] = transpose8(pl[nt][i]);
          }
        }
        if constexpr (E8) {
#pragma unroll
          for (int k2 = 0; k2 < D / 32; ++k2) {
            uint32_t w[4];
            ldsm_t(w, unit + vat[k2 & 3] + (k2 >> 2) * 128 + u * 16 * kRow);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              // a word holds two elements of two positions: an element's two positions side by side
              const uint32_t y0 = __byte_perm(w[2 * x], 0, 0x3120), y1 = __byte_perm(w[2 * x + 1], 0, 0x3120);
              const uint32_t f[4] = {widen(y0, 0), widen(y0, 1), widen(y1, 0), widen(y1, 1)};
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                M::mma(o[2 * k2 + x][nt], f, ph[nt][0], ph[nt][1]);
                M::mma(o[2 * k2 + x][nt], f, pl[nt][0], pl[nt][1]);
              }
            }
          }
        } else
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          uint32_t f[4];
          ldsm_t(f, unit + vat[kk & 3] + (kk >> 2) * 128 + u * 16 * D * 2);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            M::mma(o[kk][nt], f, ph[nt][0], ph[nt][1]);
            M::mma(o[kk][nt], f, pl[nt][0], pl[nt][1]);
          }
        }
      }
    }
    ++ct;
    if (ct < cs.nt && left > 1) continue;
    if constexpr (CL) break;

    // -- the segment, or this CTA's part of it, ends: its teams join
    const Segment done = cs;
    const bool whole = ct == done.nt && from_first, had_first = from_first;
    const int64_t g0 = end - left + 1 - ct;  // the segment's first tile in the line
    if (left > 1) {  // the next segment's queries come while this one is written
      next_segment<TREE>(a, groups, per_head, kUnit, kTile, cs);
      ct = 0;
      from_first = true;
      load_q();
    }
    sum_lanes(done.b);
    const int h0 = (done.h - done.hk * per_head) * S::kHeads;  // the segment's first head within its key head
    // a CTA has two slots: its first segment's, and that of a segment it starts and does not end
    float* to = part + (2 * (int64_t)blockIdx.x + (g0 > start ? 1 : 0)) * HT * S::kPiece;
    auto put = [&](int w, int t, const Joined& j) {  // tile t of the team's warp w
      const int nt = t / (D / 16), kk = t % (D / 16), h = w * 8 * NT + nt * 8;
      if (whole) {
        finish<T, E8, TREE>(a, done.b, g, done.hk, h0 + h, group - h0 - h, kk, j);
      } else {
        float* p = to + w * S::kPiece;
        *reinterpret_cast<float4*>(p + t * 128 + lane * 4) = j.x;
        if (kk == 0 && lane < 4) {
          *reinterpret_cast<float2*>(p + 8 * NT * D + nt * 8 + 2 * lane) = j.m;
          *reinterpret_cast<float2*>(p + 8 * NT * (D + 1) + nt * 8 + 2 * lane) = j.l;
        }
      }
    };
    if constexpr (kTeams == 1) {
#pragma unroll
      for (int t = 0; t < S::kTiles; ++t) {
        const int nt = t / (D / 16), kk = t % (D / 16);
        Joined j;
        j.x = make_float4(o[kk][nt][0], o[kk][nt][1], o[kk][nt][2], o[kk][nt][3]);
        j.m = make_float2(m[nt][0], m[nt][1]);
        j.l = make_float2(l[nt][0], l[nt][1]);
        put(hw, t, j);
      }
    } else {
      float4* mx = reinterpret_cast<float4*>(smem + S::kRing);                    // [warp][tile of the round][lane]
      float2* mm = reinterpret_cast<float2*>(mx + S::kWarps * S::kRound * 32);    // [warp][nt][lane of 4]
      float2* ml = mm + S::kWarps * NT * 4;
      if (lane < 4)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          mm[(warp * NT + nt) * 4 + lane] = make_float2(m[nt][0], m[nt][1]);
          ml[(warp * NT + nt) * 4 + lane] = make_float2(l[nt][0], l[nt][1]);
        }
#pragma unroll
      for (int t0 = 0; t0 < S::kTiles; t0 += S::kRound) {
#pragma unroll
        for (int t = t0; t < t0 + S::kRound; ++t) {
          const int nt = t / (D / 16), kk = t % (D / 16);
          mx[(warp * S::kRound + t - t0) * 32 + lane] = make_float4(o[kk][nt][0], o[kk][nt][1], o[kk][nt][2], o[kk][nt][3]);
        }
        __syncthreads();
        // a warp joins every kWarps-th of the round's tiles of all head parts
#pragma unroll
        for (int i = warp; i < HT * S::kRound; i += S::kWarps) {
          const int w = i / S::kRound, t = t0 + i % S::kRound, nt = t / (D / 16);
          Joined j;
#pragma unroll
          for (int k = 0; k < kTeams; ++k) {
            const float2 x = mm[((k * HT + w) * NT + nt) * 4 + (lane & 3)];
            j.m = make_float2(fmaxf(j.m.x, x.x), fmaxf(j.m.y, x.y));
          }
#pragma unroll
          for (int k = 0; k < kTeams; ++k)
            j.add(mm[((k * HT + w) * NT + nt) * 4 + (lane & 3)], ml[((k * HT + w) * NT + nt) * 4 + (lane & 3)],
                  mx[((k * HT + w) * S::kRound + t - t0) * 32 + lane]);
          put(w, t, j);
        }
        __syncthreads();
      }
    }
    if (by_seg && had_first && tid == 0) {
      SegMeta s{done.b, done.h, 0, 0};
      if (!whole) {
        s.pieces = deal.worker(g0 + done.nt - 1) - blockIdx.x + 1;
        s.first_slot = 2 * blockIdx.x + (g0 > start ? 1 : 0);
      }
      meta[(int64_t)done.b * groups + done.h] = s;
    }
    reset();
  }

  if constexpr (CL) {
    // -- the cluster's teams join: pieces in place of the rings
    team_sync();  // the team's last unit has been read
    constexpr int kTeamFloats = kStages * S::kUnitBytes / 4;
    float* own = reinterpret_cast<float*>(smem);
    sum_lanes(cs.b);
    store_piece(own + team * kTeamFloats + hw * S::kPiece);
    const int pieces = ranks * kTeams;
    float* wm = reinterpret_cast<float*>(smem + S::kRing);  // [piece][head]: maxima, then weights
    float* wl = wm + pieces * S::kHeads;
    cg::cluster_group cl = cg::this_cluster();
    auto piece = [&](int p, int w) {  // piece p of the team's warp w
      float* at = own + (p % kTeams) * kTeamFloats + w * S::kPiece;
      return ranks > 1 ? cl.map_shared_rank(at, p / kTeams) : at;
    };
    if (ranks > 1)
      cl.sync();
    else
      __syncthreads();
    for (int i = tid; i < pieces * S::kHeads; i += S::kThreads) {
      const int h = i % S::kHeads;
      const float* p = piece(i / S::kHeads, h / (8 * NT)) + 8 * NT * D + h % (8 * NT);
      wm[i] = p[0];
      wl[i] = p[8 * NT];
    }
    __syncthreads();
    const int h0 = (cs.h - cs.hk * per_head) * S::kHeads;
    if (tid < S::kHeads) {
      float mm = -CUDART_INF_F, sum = 0.0f;
      for (int p = 0; p < pieces; ++p) mm = fmaxf(mm, wm[p * S::kHeads + tid]);
      for (int p = 0; p < pieces; ++p) sum += piece_weight(wm[p * S::kHeads + tid], mm) * wl[p * S::kHeads + tid];
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      for (int p = 0; p < pieces; ++p) wm[p * S::kHeads + tid] = piece_weight(wm[p * S::kHeads + tid], mm) * inv;
      wl[tid] = sum == 0.0f ? 0.0f : 1.0f;  // 0: nothing attended to, whatever the values are (0 times inf is no 0)
      if (a.lse && blockIdx.x % ranks == 0 && h0 + tid < group) a.lse[lse_at<TREE>(a, cs.b, g, cs.hk, h0 + tid)] = log_sum<W>(mm, sum);
    }
    __syncthreads();
    // a warp joins tiles of 16 elements x 8 heads
    constexpr int kTiles = HT * NT * (D / 16);
    for (int t = (blockIdx.x % ranks) * S::kWarps + warp; t < kTiles; t += ranks * S::kWarps) {
      const int w = t / (NT * (D / 16)), in = t % (NT * (D / 16));
      const int h = w * 8 * NT + in / (D / 16) * 8;  // first head of the tile
      float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
      for (int p = 0; p < pieces; ++p) {
        const float4 v = reinterpret_cast<const float4*>(piece(p, w))[in * 32 + lane];
        const float2 f = *reinterpret_cast<const float2*>(wm + p * S::kHeads + h + 2 * (lane & 3));
        x.x = fmaf(f.x, v.x, x.x);
        x.y = fmaf(f.y, v.y, x.y);
        x.z = fmaf(f.x, v.z, x.z);
        x.w = fmaf(f.y, v.w, x.w);
      }
      const float2 any = *reinterpret_cast<const float2*>(wl + h + 2 * (lane & 3));
      store_tile<T, E8>((T*)a.out + cs.b * a.o_seq + row_at<TREE>(g, cs.hk, h0 + h + lane / 4, a.o_node, a.o_head), group - h0 - h,
                        in % (D / 16), x, any.x, any.y);
    }
    if (ranks > 1) cl.sync();  // the others have read this rank's pieces
  }
}

// Joins the pieces of a segment in a fixed order.  A CTA takes eight heads and
// `tiles` of their D / 16 tiles; the warps of a tile share its pieces, each
// with a running maximum, and join in shared memory.
constexpr int kJoinWarps = 8;
template <typename T, bool E8, int D, bool TREE>
__global__ void __launch_bounds__(32 * kJoinWarps)
    decode_join_kernel(DecodeArgs a, int per_head, int seg_heads, int warp_heads, int tiles, const float* part, const SegMeta* meta) {
  __shared__ float4 s_x[kJoinWarps][32];
  __shared__ float2 s_m[kJoinWarps][4], s_l[kJoinWarps][4];
  cudaGridDependencySynchronize();
  cudaTriggerProgrammaticLaunchCompletion();
  const int g = a.n_q_heads / a.c.n_heads, group = rows_of<TREE>(a, g);
  const SegMeta s = meta[blockIdx.x];
  const int h = blockIdx.y * 8, h0 = (s.head_group % per_head) * seg_heads;  // heads within the segment, and within the key head
  if (s.pieces == 0 || h0 + h >= group) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t piece_floats = warp_heads * (D + 2), slot_floats = seg_heads / warp_heads * piece_floats;
  const float* first = part + s.first_slot * slot_floats + h / warp_heads * piece_floats;
  const float* rest = part + (s.first_slot & ~1) * slot_floats + h / warp_heads * piece_floats;
  const int share = kJoinWarps / tiles;  // warps of a tile
  const int tile = blockIdx.z * tiles + warp / share;
  const int64_t x_at = (h % warp_heads / 8 * (D / 16) + tile) * 128 + lane * 4;  // the lane's part of the tile
  const int64_t m_at = (int64_t)warp_heads * D + h % warp_heads + 2 * (lane & 3);  // its two heads' maxima
  Joined j;
  j.gather<4>(warp % share, share, s.pieces, [&](int i) { return i ? rest + 2 * i * slot_floats : first; }, x_at, m_at, warp_heads);
  if (share > 1) {
    s_x[warp][lane] = j.x;
    if (lane < 4) {
      s_m[warp][lane] = j.m;
      s_l[warp][lane] = j.l;
    }
    __syncthreads();
    if (warp % share) return;
    float2 top = j.m;
    for (int w = 1; w < share; ++w) top = make_float2(fmaxf(top.x, s_m[warp + w][lane & 3].x), fmaxf(top.y, s_m[warp + w][lane & 3].y));
    j.rescale(top);
    for (int w = 1; w < share; ++w) j.add(s_m[warp + w][lane & 3], s_l[warp + w][lane & 3], s_x[warp + w][lane]);
  }
  finish<T, E8, TREE>(a, s.seq, g, s.head_group / per_head, h0 + h, group - h0 - h, tile, j);
}

constexpr int64_t kMetaBytes = (kDecodeCtas * (int64_t)sizeof(SegMeta) + 255) / 256 * 256;

// Heads of a segment for a group of query heads: up to 24 (head_dim 64: 32; 256:
// 8) in one warp, whose registers hold their accumulators, more in the warps of a
// team, which share each unit.  Measured with 256 x 2,048 positions of 2 key heads
// of 128: 20 heads 104 us in one warp of three head tiles, 112 in three warps of
// one; 16 heads 92 us in one warp, 94 in two; 32 heads 120 us in two warps of two,
// 133 in four of one, 147 in one of four, which spills.  head_dim 256, 1,024
// positions: 20 heads 130 us in three warps of one, 152 in two of two.
inline int seg_heads(int D, int group) {
  if (group <= 16) return group <= 8 ? 8 : 16;
  return group <= 24 ? 24 : group <= 32 ? 32 : 64;
}

inline int64_t decode_ws_bytes(const pe_kv_cache& c, int n_q_heads) {
  const int D = c.head_dim, n = seg_heads(D, n_q_heads / c.n_heads);
  const int64_t ctas = D == 256 ? kDecodeCtas / 2 : kDecodeCtas;
  return kMetaBytes + 2 * ctas * n * (D + 2) * 4;  // two pieces for each CTA
}

// Ranks of the cluster that takes a segment, or 0 for the line of tiles.  The
// positions that a segment can have at most (lengths are on the device) and the
// segments' number decide, so short sequences in a table of a long context take
// the line: one of 700 in a table of 32,768 14.3 us alone, 12.3 in one of 704.
// Measured with 8 key heads of 128, cluster against line: 8 sequences of 512 6.8
// against 9.5 us, 32 of 512 14.6 against 20.2, 1 of 4,096 11.0 against 10.0 (and
// a launch less on the host); beyond the bounds 128 of 256 32.4 against 30.6, 128
// of 64 16.8 against 13.5, 1 of 16,384 29.8 against 20.4.
inline int cluster_ranks(const DecodeArgs& a, int64_t segments, int tile) {
  int64_t most = (int64_t)a.c.max_pages * a.c.page_size;
  if (a.window > 0 && (int64_t)a.window + a.n_nodes + 32 < most) most = (int64_t)a.window + a.n_nodes + 32;
  const int64_t tiles = (most + tile - 1) / tile;
  if (tiles * segments > 2048 || tiles > 64 || segments > 4 * 152) return 0;
  // A larger cluster starts and joins later.  One sequence, 8 key heads, in 2, 4
  // and 8 ranks: 200 positions 5.1, 5.8, 5.8 us; 700 7.5, 6.8, 7.5; 1,500 10.5,
  // 8.5, 8.6; 3,000 16.7, 11.5, 10.1 (sixteen cost 13.0).
  const int ranks = tiles < 3 ? 1 : tiles < 10 ? 2 : tiles < 24 ? 4 : kMaxRanks;
  int r = 1;
  while (r < ranks && segments * r * 2 <= 2 * 152) r *= 2;
  return r;
}

template <typename T, bool E8, int D, int NT, int HT, bool TREE = false>
static pe_status go(const DecodeArgs& a, void* ws, cudaStream_t st) {
  using S = DecodeShape<E8, D, NT, HT>;
  const int group = a.n_q_heads / a.c.n_heads * (TREE ? a.n_nodes : 1);
  const int per_head = (group + S::kHeads - 1) / S::kHeads, groups = a.c.n_heads * per_head;
  const int64_t segments = (int64_t)a.c.n_seqs * groups;
  int shift = -1;  // of a page size that is a power of two
  if ((a.c.page_size & (a.c.page_size - 1)) == 0)
    while (a.c.page_size >> (shift + 1)) ++shift;
  const int ranks = cluster_ranks(a, segments, S::kTeams * S::kUnit);
  if (ranks) {
    auto kern = decode_attn_kernel<T, E8, D, NT, HT, true, TREE>;
    PE_TRY_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem));
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = ranks;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t lc{};
    lc.gridDim = dim3((unsigned)(segments * ranks));
    lc.blockDim = S::kThreads;
    lc.dynamicSmemBytes = S::kSmem;
    lc.stream = st;
    lc.attrs = at;
    lc.numAttrs = ranks > 1 ? 2 : 1;
    PE_TRY_CUDA(cudaLaunchKernelEx(&lc, kern, a, groups, per_head, shift, ranks, 0, false, (float*)nullptr, (SegMeta*)nullptr));
    return PE_OK;
  }
  auto kern = decode_attn_kernel<T, E8, D, NT, HT, false, TREE>;
  PE_TRY_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem));
  SegMeta* meta = reinterpret_cast<SegMeta*>(ws);
  float* part = reinterpret_cast<float*>(reinterpret_cast<char*>(ws) + kMetaBytes);
  if (segments * (((int64_t)a.c.max_pages * a.c.page_size + S::kUnit - 1) / S::kUnit + 1) / S::kCtas >= INT32_MAX - 1)
    return fail(PE_EINVAL, "n_seqs * n_heads * max_pages * page_size too large");
  const bool by_seg = segments <= S::kCtas;
  const int least = 2;  // tiles of a CTA; 4 cost a batch of 2 x 4,096 nothing, 8 14.1 us for 12.4
  PE_TRY_CUDA(launch_pdl(kern, dim3(S::kCtas), dim3(S::kThreads), S::kSmem, st, true, a, groups, per_head, shift, 0, least, by_seg, part, meta));
  // few segments have many pieces each: their tiles go to CTAs of their own
  const int heads = group < S::kHeads ? group : S::kHeads;
  const int tiles = segments <= 152 ? 1 : D == 64 ? 4 : 8;
  PE_TRY_CUDA(launch_pdl(decode_join_kernel<T, E8, D, TREE>, dim3((unsigned)(by_seg ? segments : S::kCtas), (heads + 7) / 8, D / 16 / tiles),
                         dim3(32 * kJoinWarps), 0, st, true, a, per_head, (int)S::kHeads, 8 * NT, tiles, (const float*)part, (const SegMeta*)meta));
  return PE_OK;
}

}  // namespace pe
