// Attention of one new token per sequence over a paged cache (formulas:
// pe.h).  HBM-bound: every attended key and value is read once; a position
// costs 4 D FLOP per query head, far below the tensor rate for any head count.
//
// Work is cut into tiles of 16 positions per warp team; the tiles of all
// (sequence, key head, head group) segments form one line that is dealt out
// evenly to the CTAs, so ragged lengths balance and a long cache is split
// without a plan on the host (lengths are read on the device).  A CTA whose
// range holds a whole segment writes the result; the pieces of a segment that
// crosses CTAs go to the workspace as (maximum, sum, unnormalised output) and
// a second kernel joins them in the order of the CTAs.
//
// Within a CTA each team of HT warps runs its own ring of cp.async stages, 16
// positions each; no barrier of the whole CTA is needed before a segment ends.
// Products on mma.sync, transposed: scores S^T[16 positions x 8 heads] =
// K Q^T and O^T[D x 8 heads] += V^T P^T, so that 8 query heads fill a tile's
// columns (tcgen05 wants 64 or 128 rows of queries, and a decode step has 1 to
// 16 per key head).  P enters the second product as a sum of two 16-bit
// numbers, hi + lo: one alone would add an error of the size of the result's
// own rounding.
#include <math_constants.h>

#include "tokens.cuh"

namespace pe {

constexpr int kUnit = 16;  // positions of a stage
constexpr int kDecodeCtas = 152 * 2;  // CTAs of the split at most: two on each SM

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

template <typename T>
__device__ __forceinline__ void store2(T* p, float a, float b) {
  *reinterpret_cast<uint32_t*>(p) = pack2<T>(a, b);
}

// a segment crossing CTAs, as the joining kernel finds it at its first inner
// boundary: pieces of CTAs [first, first + pieces)
struct SegMeta {
  int32_t seq, head_group, pieces, first_slot;  // pieces 0: nothing to join at this boundary
};

template <int D, int NT, int HT>
struct DecodeShape {
  // eight warps where wide heads leave one CTA on an SM and its teams have several warps
  static constexpr int kWarps = D == 256 && HT > 1 ? 8 : 4;
  static constexpr int kTeams = kWarps / HT;
  static constexpr int kCtas = D == 256 ? kDecodeCtas / 2 : kDecodeCtas;
  static constexpr int kTile = kTeams * kUnit;           // positions of a tile
  static constexpr int kHeads = 8 * NT * HT;             // query heads of a segment
  static constexpr int kUnitBytes = 2 * kUnit * D * 2;   // keys and values of a unit
  // a ring of 96 KB (two CTAs on an SM) or, for wide heads, 192 KB; at most 8 stages
  static constexpr int kFit = (D == 256 ? 196608 : 98304) / (kTeams * kUnitBytes);
  static constexpr int kStages = kFit > 8 ? 8 : kFit;
  static constexpr int kCols = NT == 2 ? 32 : D > 128 ? 128 : D;  // columns of the output joined at a time
  static constexpr int kPitch = kCols + 4;
  static constexpr int kRing = kTeams * kStages * kUnitBytes;
  static constexpr int kMerge = kTeams * kHeads * kPitch * 4;
  static constexpr int kSmem = kRing + kMerge + 2 * kTeams * kHeads * 4;
  static_assert(kMerge >= 32 * kWarps * 8, "the prefix sums of the lengths lie there first");
  static_assert(D == 256 ? kSmem <= 231000 : 2 * (kSmem + 1024 + 256) <= 233472, "shared memory of an SM");
};

struct Segment {
  int b, h;         // sequence, head group
  int nt;           // tiles
  int base, lo, n;  // position of tile 0 (a multiple of 16), attended range [lo, n)
};

__device__ __forceinline__ void seq_range(const DecodeArgs& a, int b, int tile, Segment& s) {
  const int cap = a.c.max_pages * a.c.page_size;
  s.n = min(max(a.lens[b], 0), cap);
  s.lo = a.window > 0 ? max(0, s.n - a.window) : 0;
  s.base = s.lo & ~(kUnit - 1);
  s.nt = max(1, (s.n - s.base + tile - 1) / tile);  // an empty sequence has one empty tile
}

template <typename T, int D, int NT, int HT>
__global__ void __launch_bounds__(32 * DecodeShape<D, NT, HT>::kWarps, D == 256 ? 1 : 2)
    decode_attn_kernel(DecodeArgs a, int groups, int per_head, float* part, SegMeta* meta) {
  using S = DecodeShape<D, NT, HT>;
  using M = Mma<T>;
  constexpr int kDecodeWarps = S::kWarps, kTeams = S::kTeams, kStages = S::kStages, kChunks = D / 8;
  extern __shared__ __align__(128) unsigned char smem[];
  int64_t* s_sum = reinterpret_cast<int64_t*>(smem + S::kRing);
  __shared__ int s_where[3];
  __shared__ uint32_t s_mask[kTeams][kStages];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int team = warp / HT, hw = warp % HT;
  const pe_kv_cache& c = a.c;
  const int B = c.n_seqs;

  // where this CTA's share of the tiles starts
  const int chunk = (B + 32 * kDecodeWarps - 1) / (32 * kDecodeWarps);
  {
    int64_t sum = 0;
    Segment s;
    for (int b = tid * chunk; b < min(B, (tid + 1) * chunk); ++b) {
      seq_range(a, b, S::kTile, s);
      sum += s.nt;
    }
    int64_t incl = sum;
    for (int x = 1; x < 32; x <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, incl, x);
      if (lane >= x) incl += y;
    }
    s_sum[tid] = incl;
  }
  __syncthreads();
  int64_t before = 0, total = 0;
  for (int w = 0; w < kDecodeWarps; ++w) {
    if (w < warp) before += s_sum[32 * w + 31];
    total += s_sum[32 * w + 31];
  }
  const int64_t tiles = total * groups;
  const int64_t ctas = min((int64_t)gridDim.x, tiles);
  const int64_t start = blockIdx.x * tiles / ctas, end = (blockIdx.x + 1) * tiles / ctas;
  if (blockIdx.x >= ctas) {
    if (tid == 0) meta[blockIdx.x].pieces = 0;
    return;
  }
  {
    const int64_t lo = lane ? before + s_sum[tid - 1] : before, hi = before + s_sum[tid];
    if (start >= lo * groups && start < hi * groups) {
      int64_t at = lo;
      Segment s;
      int b = tid * chunk;
      for (;; ++b) {
        seq_range(a, b, S::kTile, s);
        if (start < (at + s.nt) * groups) break;
        at += s.nt;
      }
      const int64_t in = start - at * groups;
      s_where[0] = b;
      s_where[1] = (int)(in / s.nt);
      s_where[2] = (int)(in % s.nt);
    }
  }
  __syncthreads();
  const int first_tile = s_where[2];
  Segment cs;  // the segment computed on
  cs.b = s_where[0];
  cs.h = s_where[1];
  seq_range(a, cs.b, S::kTile, cs);
  if (tid == 0) {
    // the boundary at this CTA's start joins the segment if it is the first inside it
    const int64_t g0 = start - first_tile;
    SegMeta m{cs.b, cs.h, 0, 0};
    if (first_tile > 0 && (blockIdx.x - 1) * tiles / ctas <= g0) {
      const int64_t last = ((g0 + cs.nt) * ctas + tiles - 1) / tiles - 1;  // CTA of the segment's last tile
      m.pieces = (int)(last - blockIdx.x) + 2;
      m.first_slot = 2 * (blockIdx.x - 1) + ((blockIdx.x - 1) * tiles / ctas < g0 ? 1 : 0);
    }
    meta[blockIdx.x] = m;
  }

  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + team * kStages * S::kUnitBytes;
  float* merge = reinterpret_cast<float*>(smem + S::kRing);
  float* merge_m = merge + kTeams * S::kHeads * S::kPitch;
  float* merge_l = merge_m + kTeams * S::kHeads;

  // -- loading: the tile line, kStages - 1 tiles ahead of the computation
  Segment ls = cs;
  int lt = first_tile, lstage = 0;
  int64_t lleft = end - start;
  auto load = [&]() {
    if (lleft > 0) {
      const int at = ls.base + lt * S::kTile + team * kUnit;
      const int hk = ls.h / per_head;
      // a lane finds the place of one of the unit's 16 positions
      const int pos = at + (lane & 15);
      const bool in = pos >= ls.lo && pos < ls.n;
      int page = -1;
      if (in) page = c.table[(int64_t)ls.b * c.table_stride + pos / c.page_size];
      const bool ok = page >= 0 && page < c.n_pages;
      const int64_t off = ok ? kv_page_offset(c, page) + (int64_t)(pos % c.page_size) * c.slot_stride + hk * c.head_stride : 0;
      const uint32_t mask = __ballot_sync(0xffffffffu, ok) & 0xffffu;
      if (lane == 0 && hw == 0) s_mask[team][lstage] = mask;
      constexpr int kRows = 32 / kChunks > 0 ? 32 / kChunks : 1;  // rows of one copy instruction
      constexpr int kMine = kUnit / HT;
      const uint32_t dst = ring + lstage * S::kUnitBytes;
#pragma unroll
      for (int i = 0; i < kMine / kRows; ++i) {
        const int row = hw * kMine + i * kRows + lane / kChunks;
        const int ch = lane % kChunks;
        const int64_t o = __shfl_sync(0xffffffffu, off, row) + ch * 8;
        const bool k = (mask >> row) & 1;
        const uint32_t d = dst + row * (D * 2) + ((ch ^ (row & 7)) << 4);
        copy16(d, (const T*)c.k + o, k);
        copy16(d + kUnit * D * 2, (const T*)c.v + o, k);
      }
      if (++lt == ls.nt) {
        lt = 0;
        if (++ls.h == groups) {
          ls.h = 0;
          if (++ls.b < B) seq_range(a, ls.b, S::kTile, ls);
        }
      }
      --lleft;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    lstage = lstage + 1 == kStages ? 0 : lstage + 1;
  };
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) load();

  // -- computing
  // ldmatrix places of the lane: row, and 16-byte column under the ring's
  // swizzle, whose three bits repeat every 128 bytes of a row
  uint32_t kat[4], vat[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int kr = lane & 15, vr = (lane & 7) + 8 * (lane / 16);
    kat[i] = kr * (D * 2) + (((i * 2 + lane / 16) ^ (kr & 7)) << 4);
    vat[i] = kUnit * D * 2 + vr * (D * 2) + (((i * 2 + ((lane >> 3) & 1)) ^ (vr & 7)) << 4);
  }
  const float qscale = a.scale * 1.4426950408889634f;  // scores in powers of two
  uint32_t qf[D / 16][NT][2];
  float o[D / 16][NT][4], m[NT][2], l[NT][2];
  int ct = first_tile, stage = 0, piece = 0;
  bool fresh = true;
  const int group = a.n_q_heads / c.n_heads;  // query heads of a key head
  for (int64_t left = end - start; left > 0; --left) {
    const int h0 = (cs.h % per_head) * S::kHeads;  // first head of the segment within its key head
    if (fresh) {
      const T* q = (const T*)a.q + cs.b * a.q_seq + (int64_t)(cs.h / per_head) * group * a.q_head;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int h = h0 + hw * 8 * NT + nt * 8 + lane / 4;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint32_t* p = reinterpret_cast<const uint32_t*>(q + h * a.q_head + kk * 16 + 2 * (lane & 3));
          qf[kk][nt][0] = h < group ? p[0] : 0u;
          qf[kk][nt][1] = h < group ? p[4] : 0u;
#pragma unroll
          for (int i = 0; i < 4; ++i) o[kk][nt][i] = 0.0f;
        }
        m[nt][0] = m[nt][1] = -CUDART_INF_F;
        l[nt][0] = l[nt][1] = 0.0f;
      }
      fresh = false;
    }
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
    if (HT == 1)
      __syncwarp();
    else
      asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(32 * HT) : "memory");
    load();
    const uint32_t unit = ring + stage * S::kUnitBytes;
    const uint32_t mask = s_mask[team][stage];
    stage = stage + 1 == kStages ? 0 : stage + 1;
    if (mask) {
      // two chains of products where one head tile gives only one
      constexpr int kChains = NT == 1 ? 2 : 1;
      float s[NT][4], s2[kChains][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[nt][i] = 0.0f;
        s2[kChains - 1][i] = 0.0f;
      }
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        uint32_t f[4];
        ldsm(f, unit + kat[kk & 3] + (kk >> 2) * 128);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) M::mma(kChains == 2 && (kk & 1) ? s2[1] : s[nt], f, qf[kk][nt][0], qf[kk][nt][1]);
      }
      if (kChains == 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[0][i] += s2[kChains - 1][i];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[nt][i] *= qscale;
      if (mask != 0xffffu) {
        const bool r0 = (mask >> (lane / 4)) & 1, r1 = (mask >> (lane / 4 + 8)) & 1;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          if (!r0) s[nt][0] = s[nt][1] = -CUDART_INF_F;
          if (!r1) s[nt][2] = s[nt][3] = -CUDART_INF_F;
        }
      }
      // the reference of the exponentials follows the maximum only when it is
      // passed by 8 (a factor of 256): few units rescale
      bool over = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) over |= s[nt][i] > m[nt][i & 1] + 8.0f;
      if (__any_sync(0xffffffffu, over)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float x = fmaxf(s[nt][i], s[nt][i + 2]);
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
            x = fmaxf(x, m[nt][i]);
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
      uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float r0 = (m[nt][0] == -CUDART_INF_F ? 0.0f : m[nt][0]) - M::kBias;
        const float r1 = (m[nt][1] == -CUDART_INF_F ? 0.0f : m[nt][1]) - M::kBias;
        const float p0 = exp2_fast(s[nt][0] - r0), p1 = exp2_fast(s[nt][1] - r1);
        const float p2 = exp2_fast(s[nt][2] - r0), p3 = exp2_fast(s[nt][3] - r1);
        l[nt][0] += p0 + p2;
        l[nt][1] += p1 + p3;
        split2<T>(p0, p1, ph[nt][0], pl[nt][0]);
        split2<T>(p2, p3, ph[nt][1], pl[nt][1]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          ph[nt][i] = transpose8(ph[nt][i]);
          pl[nt][i] = transpose8(pl[nt][i]);
        }
      }
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        uint32_t f[4];
        ldsm_t(f, unit + vat[kk & 3] + (kk >> 2) * 128);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          M::mma(o[kk][nt], f, ph[nt][0], ph[nt][1]);
          M::mma(o[kk][nt], f, pl[nt][0], pl[nt][1]);
        }
      }
    }
    ++ct;
    if (ct < cs.nt && left > 1) continue;

    // -- the segment, or this CTA's part of it, ends: join the teams
    const bool whole = ct == cs.nt && (piece > 0 || first_tile == 0);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float x = l[nt][i];
        x += __shfl_xor_sync(0xffffffffu, x, 4);
        x += __shfl_xor_sync(0xffffffffu, x, 8);
        x += __shfl_xor_sync(0xffffffffu, x, 16);
        if (lane < 4) {
          const int h = team * S::kHeads + hw * 8 * NT + nt * 8 + 2 * lane + i;
          merge_m[h] = m[nt][i];
          merge_l[h] = x;
        }
      }
    const int heads = min(S::kHeads, group - h0);
    const int64_t slot = 2 * (int64_t)blockIdx.x + (piece > 0 ? 1 : 0);
    float* po = part + slot * S::kHeads * (D + 2);
    const int64_t head = (int64_t)(cs.h / per_head) * group + h0;
#pragma unroll
    for (int c0 = 0; c0 < D; c0 += S::kCols) {
#pragma unroll
      for (int kk = c0 / 16; kk < (c0 + S::kCols) / 16; ++kk)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int h = team * S::kHeads + hw * 8 * NT + nt * 8 + 2 * (lane & 3) + (i & 1);
            merge[h * S::kPitch + kk * 16 - c0 + lane / 4 + (i >> 1) * 8] = o[kk][nt][i];
          }
      __syncthreads();
      for (int i = tid; i < heads * (S::kCols / 2); i += 32 * kDecodeWarps) {
        const int h = i / (S::kCols / 2), d = (i % (S::kCols / 2)) * 2;
        float mm = -CUDART_INF_F;
#pragma unroll
        for (int t = 0; t < kTeams; ++t) mm = fmaxf(mm, merge_m[t * S::kHeads + h]);
        float x = 0.0f, y = 0.0f, sum = 0.0f;
#pragma unroll
        for (int t = 0; t < kTeams; ++t) {
          const float mt = merge_m[t * S::kHeads + h];
          // a team that met nothing has sum 0; a NaN of any kind stays
          const float f = mt == -CUDART_INF_F ? (mm == -CUDART_INF_F ? 1.0f : 0.0f) : exp2_fast(mt - mm);
          const float2 v = *reinterpret_cast<const float2*>(&merge[(t * S::kHeads + h) * S::kPitch + d]);
          sum += f * merge_l[t * S::kHeads + h];
          x += f * v.x;
          y += f * v.y;
        }
        if (whole) {
          const float inv = 1.0f / sum;
          store2((T*)a.out + cs.b * a.o_seq + (head + h) * a.o_head + c0 + d, sum == 0.0f ? 0.0f : x * inv, sum == 0.0f ? 0.0f : y * inv);
          if (c0 == 0 && d == 0 && a.lse)
            a.lse[(int64_t)cs.b * a.n_q_heads + head + h] =
                sum == 0.0f ? -CUDART_INF_F : (mm == -CUDART_INF_F ? 0.0f : mm - M::kBias) * 0.69314718f + logf(sum);
        } else {
          *reinterpret_cast<float2*>(po + h * D + c0 + d) = make_float2(x, y);
          if (c0 == 0 && d == 0) {
            po[S::kHeads * D + h] = mm;
            po[S::kHeads * (D + 1) + h] = sum;
          }
        }
      }
      __syncthreads();
    }
    ++piece;
    fresh = true;
    if (ct == cs.nt) {
      ct = 0;
      if (++cs.h == groups) {
        cs.h = 0;
        if (++cs.b < B && left > 1) seq_range(a, cs.b, S::kTile, cs);
      }
    }
  }
}

// joins the pieces of one segment, in the order of the CTAs: one CTA per
// boundary and head
template <typename T, int D>
__global__ void __launch_bounds__(D / 2) decode_join_kernel(DecodeArgs a, int per_head, int seg_heads, const float* part, const SegMeta* meta) {
  const SegMeta s = meta[blockIdx.x];
  const int group = a.n_q_heads / a.c.n_heads;
  const int h = blockIdx.y, h0 = (s.head_group % per_head) * seg_heads;
  if (s.pieces == 0 || h0 + h >= group) return;
  const int64_t size = (int64_t)seg_heads * (D + 2);
  const int d = threadIdx.x * 2;
  // slots of the pieces: the first CTA's own, then the first one of each CTA after it
  const int64_t second = 2 * (int64_t)blockIdx.x;
  float mm = -CUDART_INF_F;
  for (int i = 0; i < s.pieces; ++i) {
    const float* p = part + (i ? second + 2 * (i - 1) : s.first_slot) * size;
    mm = fmaxf(mm, p[seg_heads * D + h]);
  }
  float x = 0.0f, y = 0.0f, sum = 0.0f;
  for (int i = 0; i < s.pieces; ++i) {
    const float* p = part + (i ? second + 2 * (i - 1) : s.first_slot) * size;
    const float mt = p[seg_heads * D + h];
    const float f = mt == -CUDART_INF_F ? (mm == -CUDART_INF_F ? 1.0f : 0.0f) : exp2_fast(mt - mm);
    const float2 v = *reinterpret_cast<const float2*>(p + h * D + d);
    sum += f * p[seg_heads * (D + 1) + h];
    x += f * v.x;
    y += f * v.y;
  }
  const float inv = 1.0f / sum;
  const int64_t head = (int64_t)(s.head_group / per_head) * group + h0 + h;
  store2((T*)a.out + s.seq * a.o_seq + head * a.o_head + d, sum == 0.0f ? 0.0f : x * inv, sum == 0.0f ? 0.0f : y * inv);
  if (d == 0 && a.lse)
    a.lse[(int64_t)s.seq * a.n_q_heads + head] =
        sum == 0.0f ? -CUDART_INF_F : (mm == -CUDART_INF_F ? 0.0f : mm - Mma<T>::kBias) * 0.69314718f + logf(sum);
}

constexpr int64_t kMetaBytes = (kDecodeCtas * (int64_t)sizeof(SegMeta) + 255) / 256 * 256;

// heads of a segment for a group of query heads: 8, or 16 in one warp; 32 and
// 64 in the two or four warps of a team, which share each unit
static int seg_heads(int group) { return group <= 8 ? 8 : group <= 16 ? 16 : group <= 32 ? 32 : 64; }

int64_t decode_attn_ws_bytes(const pe_kv_cache& c, int n_q_heads) {
  return kMetaBytes + 2 * kDecodeCtas * (int64_t)seg_heads(n_q_heads / c.n_heads) * (c.head_dim + 2) * 4;
}

template <typename T, int D, int NT, int HT>
static pe_status go(const DecodeArgs& a, void* ws, cudaStream_t st) {
  using S = DecodeShape<D, NT, HT>;
  auto kern = decode_attn_kernel<T, D, NT, HT>;
  PE_TRY_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem));
  const int group = a.n_q_heads / a.c.n_heads;
  const int per_head = (group + S::kHeads - 1) / S::kHeads;
  SegMeta* meta = reinterpret_cast<SegMeta*>(ws);
  float* part = reinterpret_cast<float*>(reinterpret_cast<char*>(ws) + kMetaBytes);
  kern<<<S::kCtas, 32 * S::kWarps, S::kSmem, st>>>(a, a.c.n_heads * per_head, per_head, part, meta);
  PE_CHECK_LAUNCH("decode_attn");
  decode_join_kernel<T, D><<<dim3(S::kCtas, S::kHeads < group ? S::kHeads : group), D / 2, 0, st>>>(a, per_head, S::kHeads, part, meta);
  PE_CHECK_LAUNCH("decode_join");
  return PE_OK;
}

template <typename T, int D>
static pe_status go_heads(const DecodeArgs& a, void* ws, cudaStream_t st) {
  const int n = seg_heads(a.n_q_heads / a.c.n_heads);
  if (n == 8) return go<T, D, 1, 1>(a, ws, st);
  if (n == 16) return go<T, D, 2, 1>(a, ws, st);
  if (n == 32) return go<T, D, 2, 2>(a, ws, st);
  return go<T, D, 2, 4>(a, ws, st);
}

template <typename T>
static pe_status go_dim(const DecodeArgs& a, void* ws, cudaStream_t st) {
  if (a.c.head_dim == 64) return go_heads<T, 64>(a, ws, st);
  if (a.c.head_dim == 128) return go_heads<T, 128>(a, ws, st);
  return go_heads<T, 256>(a, ws, st);
}

pe_status decode_attn_launch(const DecodeArgs& a, void* ws, cudaStream_t st) {
  ProfScope ps(PE_PROF_DECODE_ATTN, st);
  return a.c.dtype == PE_BF16 ? go_dim<__nv_bfloat16>(a, ws, st) : go_dim<__half>(a, ws, st);
}

}  // namespace pe
