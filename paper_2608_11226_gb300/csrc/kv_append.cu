// Keys and values of new tokens into a paged cache of 16 or 8 bits; queries and
// keys are rotated by their position on the way (formulas: pe.h).  HBM-bound:
// each row is read and written once, two FMAs an element.
//
// A lane holds one item of a head, two 16-byte chunks whose elements pair up
// under the rotation, and keeps its cosines and sines while it goes through
// the token's heads (query heads, key heads, value heads in one line); the
// chunks of kAhead heads are in flight at a time: three, with five CTAs on an
// SM (32,768 tokens of 64 + 16 heads of 128: 201 us, the copy rate; four with four
// CTAs took 1% longer, two with eight 3%).
//
// Into an 8-bit cache a row's lanes find its largest element with shuffles and
// take the scale from that one's exponent and mantissa: no division, and every
// quotient is exact until it becomes a code (32,768 tokens of 64 + 16 heads of
// 128: 199 us, 95% of the copy rate; 32 tokens 2.2 us).
#include "tokens.cuh"

namespace pe {

constexpr int kAppendWarps = 4, kAhead = 3;

// codes of four elements times a power of two
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float f) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b * f), "f"(a * f));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d * f), "f"(c * f));
  return (uint32_t)lo | (uint32_t)hi << 16;
}

// E8: an 8-bit cache
template <typename T, int D, bool E8>
__global__ void __launch_bounds__(32 * kAppendWarps, 5)
    kv_append_kernel(pe_kv_cache c, pe_kv_scales sc, pe_kv_tokens t, const int32_t* slots, int steps) {
  constexpr int kItems = D / 16, kHeads = 32 / kItems;  // items of a head; heads of a step
  const int lane = threadIdx.x & 31, item = lane % kItems, sub = lane / kItems;
  const int64_t tok = (int64_t)blockIdx.x * kAppendWarps + threadIdx.x / 32;
  pdl_enter();
  if (tok >= t.n_tokens) return;
  const int nq = t.q ? t.n_q_heads : 0, nk = c.n_heads, heads = nq + 2 * nk;
  const int p = t.pos[tok], at = slots ? slots[tok] : p;
  const int s = t.seq ? t.seq[tok] : (int)tok;
  const int rot = t.rot_dim;
  // chunks of the item, and whether they turn: pairs (i, i + rot/2) or neighbours
  const bool turn = item < rot / 16;
  const int c0 = t.interleaved || !turn ? 2 * item : item;
  const int c1 = t.interleaved || !turn ? c0 + 1 : item + rot / 16;

  // the first heads are on their way before the position is known
  const int begin = blockIdx.y * steps * kHeads + sub, end = min(heads, (int)(blockIdx.y + 1) * steps * kHeads);
  uint4 x[kAhead], y[kAhead];
  auto fetch = [&](int h0) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int h = h0 + u * kHeads;
      if (h >= end) break;
      const T* src = h < nq        ? (const T*)t.q + tok * t.q_token_stride + h * t.q_head_stride
                     : h < nq + nk ? (const T*)t.k + tok * t.k_token_stride + (h - nq) * t.k_head_stride
                                   : (const T*)t.v + tok * t.v_token_stride + (h - nq - nk) * t.v_head_stride;
      x[u] = *reinterpret_cast<const uint4*>(src + c0 * 8);
      y[u] = *reinterpret_cast<const uint4*>(src + c1 * 8);
    }
  };
  fetch(begin);

  const bool live = p >= 0 && at >= 0 && at < c.max_pages * c.page_size && (rot == 0 || p < t.max_pos) && s >= 0 && s < c.n_seqs;
  int64_t slot = -1, sslot = 0;
  if (live) {
    const int page = c.table[(int64_t)s * c.table_stride + at / c.page_size];
    if (page >= 0 && page < c.n_pages) {
      slot = kv_page_offset(c, page) + (int64_t)(at % c.page_size) * c.slot_stride;
      if (E8) sslot = page * sc.page_stride + (int64_t)(at % c.page_size) * sc.slot_stride;
    }
  }
  float co[8], si[8];
  if (live && turn) {
    const float4* r = reinterpret_cast<const float4*>(t.rot + (int64_t)p * rot + 8 * item);
    const float4 a = r[0], b = r[1], x = r[rot / 8], y = r[rot / 8 + 1];
    co[0] = a.x, co[1] = a.y, co[2] = a.z, co[3] = a.w, co[4] = b.x, co[5] = b.y, co[6] = b.z, co[7] = b.w;
    si[0] = x.x, si[1] = x.y, si[2] = x.z, si[3] = x.w, si[4] = y.x, si[5] = y.y, si[6] = y.z, si[7] = y.w;
  }

  for (int h0 = begin; h0 < end; h0 += kAhead * kHeads) {
    if (h0 != begin) fetch(h0);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int h = h0 + u * kHeads;
      if (h >= end) break;
      if constexpr (E8) {
        if (h >= nq) {
          if (slot < 0) continue;
          const bool key = h < nq + nk;
          const int hk = key ? h - nq : h - nq - nk;
          float f[8], g[8];  // the item's elements, chunk by chunk
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 a = unpack2<T>(reinterpret_cast<const uint32_t*>(&x[u])[i]), b = unpack2<T>(reinterpret_cast<const uint32_t*>(&y[u])[i]);
            f[2 * i] = a.x, f[2 * i + 1] = a.y, g[2 * i] = b.x, g[2 * i + 1] = b.y;
          }
          if (turn && key) {
            // products and sums rounded one by one: codes do not depend on how they are contracted
            auto pair = [](float& a, float& b, float co, float si) {
              const float p = __fsub_rn(__fmul_rn(a, co), __fmul_rn(b, si));
              b = __fadd_rn(__fmul_rn(b, co), __fmul_rn(a, si));
              a = p;
            };
            if (t.interleaved) {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                pair(f[2 * i], f[2 * i + 1], co[i], si[i]);
                pair(g[2 * i], g[2 * i + 1], co[4 + i], si[4 + i]);
              }
            } else {
#pragma unroll
              for (int i = 0; i < 8; ++i) pair(f[i], g[i], co[i], si[i]);
            }
          }
          uint32_t most = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) most = max(most, max(__float_as_uint(f[i]) & 0x7fffffffu, __float_as_uint(g[i]) & 0x7fffffffu));
          const uint32_t members = (kItems == 32 ? 0xffffffffu : (1u << kItems) - 1) << (lane & ~(kItems - 1));  // the head's lanes
#pragma unroll
          for (int w = 1; w < kItems; w *= 2) most = max(most, __shfl_xor_sync(members, most, w));
          // 448 = 1.75 * 2^8: one more than the exponent less 8 where the mantissa is above 1.75
          const int byte = most >= 0x7f800000u ? 255 : max((int)(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u), 63);
          const float inv = __uint_as_float((254u - byte) << 23);  // 2^-e
          uint8_t* to = (uint8_t*)(key ? c.k : c.v) + slot + hk * c.head_stride;
          uint2 a = make_uint2(codes4(f[0], f[1], f[2], f[3], inv), codes4(f[4], f[5], f[6], f[7], inv));
          uint2 b = make_uint2(codes4(g[0], g[1], g[2], g[3], inv), codes4(g[4], g[5], g[6], g[7], inv));
          if (byte == 255) a = b = make_uint2(0, 0);
          *reinterpret_cast<uint2*>(to + c0 * 8) = a;
          *reinterpret_cast<uint2*>(to + c1 * 8) = b;
          if (item == 0) (key ? sc.k : sc.v)[sslot + hk * sc.head_stride] = (uint8_t)byte;
          continue;
        }
      }
      T* dst;
      if (h < nq)
        dst = (T*)t.q_out + tok * t.q_out_token_stride + h * t.q_out_head_stride;
      else if (slot < 0)
        continue;
      else
        dst = h < nq + nk ? (T*)c.k + slot + (h - nq) * c.head_stride : (T*)c.v + slot + (h - nq - nk) * c.head_stride;
      if (!live) {
        x[u] = y[u] = make_uint4(0, 0, 0, 0);
      } else if (turn && h < nq + nk) {
        uint32_t* a = reinterpret_cast<uint32_t*>(&x[u]);
        uint32_t* b = reinterpret_cast<uint32_t*>(&y[u]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 f = unpack2<T>(a[i]), g = unpack2<T>(b[i]);
          if (t.interleaved) {
            a[i] = pack2<T>(f.x * co[i] - f.y * si[i], f.y * co[i] + f.x * si[i]);
            b[i] = pack2<T>(g.x * co[4 + i] - g.y * si[4 + i], g.y * co[4 + i] + g.x * si[4 + i]);
          } else {
            a[i] = pack2<T>(f.x * co[2 * i] - g.x * si[2 * i], f.y * co[2 * i + 1] - g.y * si[2 * i + 1]);
            b[i] = pack2<T>(g.x * co[2 * i] + f.x * si[2 * i], g.y * co[2 * i + 1] + f.y * si[2 * i + 1]);
          }
        }
      }
      *reinterpret_cast<uint4*>(dst + c0 * 8) = x[u];
      *reinterpret_cast<uint4*>(dst + c1 * 8) = y[u];
    }
  }
}

template <typename T, int D, bool E8>
static pe_status go(const pe_kv_cache& c, const pe_kv_scales& sc, const pe_kv_tokens& t, const int32_t* slots, cudaStream_t st) {
  constexpr int kHeads = 32 / (D / 16);
  const int heads = (t.q ? t.n_q_heads : 0) + 2 * c.n_heads;
  const int all = ceil_div(heads, kHeads);  // steps of a token
  // a warp takes whole tokens where there are enough of them for 16 warps on
  // each SM; fewer tokens are split by heads
  const int64_t want = ceil_div(152 * 16, t.n_tokens);
  const int parts = (int)(want < all ? want : all), steps = ceil_div(all, parts);
  PE_TRY_CUDA(launch_pdl(kv_append_kernel<T, D, E8>, dim3((unsigned)ceil_div(t.n_tokens, kAppendWarps), ceil_div(all, steps)),
                         dim3(32 * kAppendWarps), 0, st, true, c, sc, t, slots, steps));
  return PE_OK;
}

template <typename T, bool E8>
static pe_status go_dim(const pe_kv_cache& c, const pe_kv_scales& sc, const pe_kv_tokens& t, const int32_t* slots, cudaStream_t st) {
  if (c.head_dim == 64) return go<T, 64, E8>(c, sc, t, slots, st);
  if (c.head_dim == 128) return go<T, 128, E8>(c, sc, t, slots, st);
  return go<T, 256, E8>(c, sc, t, slots, st);
}

pe_status kv_append_launch(const pe_kv_cache& c, const pe_kv_scales& sc, const pe_kv_tokens& t, const int32_t* slots, int dtype,
                           cudaStream_t st) {
  ProfScope ps(PE_PROF_KV_APPEND, st);
  if (c.dtype == PE_E4M3)
    return dtype == PE_BF16 ? go_dim<__nv_bfloat16, true>(c, sc, t, slots, st) : go_dim<__half, true>(c, sc, t, slots, st);
  return dtype == PE_BF16 ? go_dim<__nv_bfloat16, false>(c, sc, t, slots, st) : go_dim<__half, false>(c, sc, t, slots, st);
}

// ---------------------------------------------------------------------------
// Rows from one position of a sequence to another.  A CTA holds all moves of one
// sequence's heads, or of some of them, keys or values, in registers between the
// reads and the writes, so that a move's source may be another's target.  Bound
// by latency: three dependent reads, then the write (32 sequences of 5 moves, 8
// heads of 128: 5.7 us); with as many heads a CTA as its threads hold 16-byte
// parts for, 512 sequences of 16 moves of 16 heads of 128 codes take 15.0 us
// (a head a CTA: 19.2).
// ---------------------------------------------------------------------------
constexpr int kMoveThreads = 256, kMoveMost = 64;

// R: bytes of a row; kEach: 16-byte parts of a thread
template <int R, int kEach>
__global__ void __launch_bounds__(kMoveThreads) kv_move_kernel(MoveArgs a, int heads) {
  constexpr int kChunks = R / 16;
  const pe_kv_cache& c = a.c;
  const int b = blockIdx.x, h0 = blockIdx.y * heads, ch = threadIdx.x % kChunks;
  const bool value = blockIdx.z != 0, eight = c.dtype == PE_E4M3;
  const int es = eight ? 1 : 2;  // bytes of an element
  pdl_enter();
  char* base = (char*)(value ? c.v : c.k) + ch * 16;
  uint8_t* scales = value ? a.sc.v : a.sc.k;
  const int cap = c.max_pages * c.page_size;
  uint4 x[kEach];
  uint8_t sx[kEach];
  int64_t to[kEach], sto[kEach];  // offsets of the target and of its scale; -1: no move
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int r = (threadIdx.x + i * kMoveThreads) / kChunks, h = r / a.n, m = r - h * a.n;  // of n moves of each head
    to[i] = -1;
    sto[i] = 0;
    x[i] = make_uint4(0, 0, 0, 0);
    sx[i] = 0;
    if (h >= heads || h0 + h >= c.n_heads) continue;
    const int s = a.src[b * a.src_stride + m], d = a.dst[b * a.dst_stride + m];
    if (s < 0 || s >= cap || d < 0 || d >= cap || s == d) continue;
    const int32_t* table = c.table + (int64_t)b * c.table_stride;
    const int si = s / c.page_size, di = d / c.page_size;
    const int sp = table[si], dp = table[di];
    if (sp < 0 || sp >= c.n_pages || dp < 0 || dp >= c.n_pages) continue;
    const int64_t head = (h0 + h) * c.head_stride, shead = (h0 + h) * a.sc.head_stride;
    const int ss = s - si * c.page_size, ds = d - di * c.page_size;
    to[i] = (kv_page_offset(c, dp) + (int64_t)ds * c.slot_stride + head) * es;
    x[i] = *reinterpret_cast<const uint4*>(base + (kv_page_offset(c, sp) + (int64_t)ss * c.slot_stride + head) * es);
    if (eight && ch == 0) {
      sto[i] = dp * a.sc.page_stride + (int64_t)ds * a.sc.slot_stride + shead;
      sx[i] = scales[sp * a.sc.page_stride + (int64_t)ss * a.sc.slot_stride + shead];
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    if (to[i] < 0) continue;
    *reinterpret_cast<uint4*>(base + to[i]) = x[i];
    if (eight && ch == 0) scales[sto[i]] = sx[i];
  }
}

template <int R>
static pe_status move_rows(const MoveArgs& a, cudaStream_t st) {
  constexpr int kChunks = R / 16, kMany = kMoveMost * kChunks / kMoveThreads > 4 ? kMoveMost * kChunks / kMoveThreads : 4;
  // as many heads as four parts a thread allow, fewer where that leaves SMs without a CTA
  int heads = kMoveThreads * 4 / (a.n * kChunks);
  heads = heads < 1 ? 1 : heads > a.c.n_heads ? a.c.n_heads : heads;
  while (heads > 1 && (int64_t)a.c.n_seqs * ceil_div(a.c.n_heads, heads) * 2 < 2 * 152) heads = (heads + 1) / 2;
  const dim3 grid(a.c.n_seqs, ceil_div(a.c.n_heads, heads), 2), block(kMoveThreads);
  const int parts = ceil_div((int64_t)a.n * kChunks * heads, kMoveThreads);
  if (parts <= 1)
    PE_TRY_CUDA(launch_pdl(kv_move_kernel<R, 1>, grid, block, 0, st, true, a, heads));
  else if (parts <= 4)
    PE_TRY_CUDA(launch_pdl(kv_move_kernel<R, 4>, grid, block, 0, st, true, a, heads));
  else
    PE_TRY_CUDA(launch_pdl(kv_move_kernel<R, kMany>, grid, block, 0, st, true, a, heads));
  return PE_OK;
}

pe_status kv_move_launch(const MoveArgs& a, cudaStream_t st) {
  ProfScope ps(PE_PROF_KV_MOVE, st);
  const int row = a.c.head_dim * (a.c.dtype == PE_E4M3 ? 1 : 2);
  return row == 64 ? move_rows<64>(a, st) : row == 128 ? move_rows<128>(a, st) : row == 256 ? move_rows<256>(a, st) : move_rows<512>(a, st);
}

}  // namespace pe
