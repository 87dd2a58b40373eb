// Keys and values of new tokens into a paged cache; queries and keys are
// rotated by their position on the way (formulas: pe.h).  HBM-bound: each row
// is read and written once, two FMAs an element.
//
// A lane holds one item of a head, two 16-byte chunks whose elements pair up
// under the rotation, and keeps its cosines and sines while it goes through
// the token's heads (query heads, key heads, value heads in one line); the
// chunks of kAhead heads are in flight at a time: three, with five CTAs on an
// SM (32,768 tokens of 64 + 16 heads of 128: 201 us, the copy rate; four with four
// CTAs took 1% longer, two with eight 3%).
#include "tokens.cuh"

namespace pe {

constexpr int kAppendWarps = 4, kAhead = 3;

template <typename T, int D>
__global__ void __launch_bounds__(32 * kAppendWarps, 5) kv_append_kernel(pe_kv_cache c, pe_kv_tokens t, int steps) {
  constexpr int kItems = D / 16, kHeads = 32 / kItems;  // items of a head; heads of a step
  const int lane = threadIdx.x & 31, item = lane % kItems, sub = lane / kItems;
  const int64_t tok = (int64_t)blockIdx.x * kAppendWarps + threadIdx.x / 32;
  pdl_enter();
  if (tok >= t.n_tokens) return;
  const int nq = t.q ? t.n_q_heads : 0, nk = c.n_heads, heads = nq + 2 * nk;
  const int p = t.pos[tok];
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

  const bool live = p >= 0 && p < c.max_pages * c.page_size && (rot == 0 || p < t.max_pos) && s >= 0 && s < c.n_seqs;
  int64_t slot = -1;
  if (live) {
    const int page = c.table[(int64_t)s * c.table_stride + p / c.page_size];
    if (page >= 0 && page < c.n_pages) slot = kv_page_offset(c, page) + (int64_t)(p % c.page_size) * c.slot_stride;
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

template <typename T, int D>
static pe_status go(const pe_kv_cache& c, const pe_kv_tokens& t, cudaStream_t st) {
  constexpr int kHeads = 32 / (D / 16);
  const int heads = (t.q ? t.n_q_heads : 0) + 2 * c.n_heads;
  const int all = ceil_div(heads, kHeads);  // steps of a token
  // a warp takes whole tokens where there are enough of them for 16 warps on
  // each SM; fewer tokens are split by heads
  const int64_t want = ceil_div(152 * 16, t.n_tokens);
  const int parts = (int)(want < all ? want : all), steps = ceil_div(all, parts);
  PE_TRY_CUDA(launch_pdl(kv_append_kernel<T, D>, dim3((unsigned)ceil_div(t.n_tokens, kAppendWarps), ceil_div(all, steps)),
                         dim3(32 * kAppendWarps), 0, st, true, c, t, steps));
  return PE_OK;
}

template <typename T>
static pe_status go_dim(const pe_kv_cache& c, const pe_kv_tokens& t, cudaStream_t st) {
  if (c.head_dim == 64) return go<T, 64>(c, t, st);
  if (c.head_dim == 128) return go<T, 128>(c, t, st);
  return go<T, 256>(c, t, st);
}

pe_status kv_append_launch(const pe_kv_cache& c, const pe_kv_tokens& t, cudaStream_t st) {
  ProfScope ps(PE_PROF_KV_APPEND, st);
  return c.dtype == PE_BF16 ? go_dim<__nv_bfloat16>(c, t, st) : go_dim<__half>(c, t, st);
}

}  // namespace pe
