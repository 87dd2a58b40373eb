// Attention of one or several new tokens over a paged cache of 16 or 8 bits on
// tcgen05 (formulas: pe.h).
//
// A sequence's new tokens and the query heads of a key head are the rows of one
// matrix, so keys and values are read once for all of them: S = Q K^T and
// O += P V are products of 128 rows with tiles of kKeys positions.  Up to 128
// rows the cache's bytes bound it (bf16, head_dim 128: 1,536 clk of products against
// 2,790 of HBM for 128 positions), beyond 256 the products and the exponentials do.
//
// One CTA on an SM.  Tiles of all (sequence, key head, block of rows) segments
// form one line that is dealt out evenly to the CTAs; a segment that crosses CTAs
// leaves pieces (unnormalised output, maxima, sums) that a second kernel joins in
// the order of the CTAs.  A segment's end (the last output waited for, 128 rows
// stored) takes 6-9 k clk, in which little else goes on: in the dealing it counts
// as kTurn tiles (64 x up to 8,192 positions: 208 us for 250 without).
//
// Roles of the 16 warps; what one waits for never holds up another's work:
//   0-7    softmax: a thread reads its row of S from TMEM and puts the weights P
//          back as the second product's operand
//   8      issues the products
//   9, 10  places: page of each position, offsets, masks, some tiles ahead (table
//          entries are on their way three turns before; 8 bits: one warp)
//   11     queries (16 bits)
//   10, 11 scales of keys and of values, and copies of the codes to stages (8 bits)
//   12-15  bring entries into the ring that the products read: 16 bits by cp.async
//          from whatever pages, two warps keys and two values; 8 bits from the
//          stages through registers, where codes become fp16
// A role's code is kept short: together they pass the instruction cache, which was
// what cost most (whole tiles without masks, loops not unrolled: 549 to 510 us for 512
// rows over 8 bits; what rarely runs in functions of its own: 483 to 416).  Tensor copies of a page's rows in place of cp.async gave nothing
// for 16 bits; a bulk copy for each row of 8 bits took 36 clk each (524 us for 208 with 32
// rows and 32,640 positions).  There a tile takes 3.7 k clk: a scale warp's loop, 1.6 k of
// it copies at the rate of cp.async (22 clk an instruction of a warp), and next to it
// 2.9 k of widening.  Up to 64 rows the softmax needs four warps; the others as widening
// warps (235 us for 208) or copying apart from the scales (229) made it slower, and so did more
// copies at once: what they share is the path to shared memory.
//   Wide (more than 128 rows in a block): each warpgroup has 128 rows of its own,
//     whose products run while the other works on its weights; P replaces S.  (Tiles of
//     64 positions, with two buffers of S, were as fast at best: what a tile costs
//     besides its products came twice as often.)
//   Narrow: both warpgroups share one tile of 128 rows, half of the tile's columns
//     each (they exchange the maxima), and S, which P replaces, has two buffers.
//
// Measured, 8 sequences of 32,640 positions, 8 key heads: 16 bits, head_dim 128, 128
// rows a key head 194 us (5.5 TB/s, 81% of the copy rate), 256 rows 293; head_dim 256, 128
// rows 366 (87%).  8 bits, head_dim 128, 128 rows 249 us, 256 rows 315: there the
// warps that widen codes and the softmax set the pace (issue active 35%, 14%
// of the stalls for instructions).
//
// An 8-bit row is its codes times 2^e.  Where rows attend differently, or scales lie far
// apart, the products are of the codes themselves, exact in fp16; a key's scale multiplies its
// column of scores and a value's exponent is added to it, so that the running maximum is
// that of weight times scale, and the sum of the weights takes the value's scale out again.  A row's
// scale so counts for that row alone, and for those who attend to it.  Reading three numbers a
// column for every row is dear (256 rows, 8 sequences of 32,640 positions: 564 us for 314), so
// where everyone attends to the whole tile and its exponents are close to the largest, E, codes become
// fp16 as code * 2^(e - E), which is exact, and 2^E goes into the exponentials' argument: keys within
// 14 of E, values within 5, because E stands for their exponents in the running maximum.
// Queries become fp16 with a power of two of their own: exact for fp16,
// for bf16 down to 2^-31 of the row's largest (the rest is off by 2^-39 of that at most).
//
// P enters the second product as a sum of two 16-bit numbers, hi + lo (bf16, or fp16 over
// fp16 and 8 bits), which leave 2^-18 (fp16: 2^-24) of a weight, as on the one-token kernel: the
// result is as exact as its own rounding for any number of rows.  (One number alone: 2.0e-3
// in the relative 2-norm for 1.6e-3 in bf16, 2.8e-4 for 2.1e-4 in fp16.)  Both parts lie where the
// scores of their keys were.  The second product and the splitting cost, with 8 sequences of
// 32,640 positions and 128 rows over 16 bits, 127 to 153 us (head_dim 64), 184 to 194 (128), 350 to 366
// (256), and 237 to 293 with 256 rows of 128.
// With bf16 queries over 8 bits P is one fp16 number: off by 2^-12 of a weight at most, where the
// result's rounding is off by up to 2^-8 (the low part costs fp16 queries 249 to 299 us, 256 rows 315 to 423).
// Sums of weights are of the fp32 weights.
//
// Weights are relative to a running maximum that follows only when it is passed
// by 8 (a factor of 256), so the output is seldom rescaled.
#pragma once

#include <math_constants.h>

#include <type_traits>

#include "tc.cuh"
#include "tokens.cuh"

namespace pe {
namespace tree {

constexpr int kCtas = 152;
constexpr int kInfos = 16;  // tiles whose description is kept: what the ring holds, and what is placed ahead

struct SegMeta {
  int32_t seq, group, pieces, first_slot;  // pieces 0: nothing to join
};

template <int D, bool E8, bool WIDE>
struct Shape {
  static_assert(!(WIDE && D == 256), "two outputs of 256 columns leave no room for scores");
  static constexpr int kKeys = D == 256 ? 64 : 128;
  static constexpr int kBufs = WIDE ? 1 : 2;  // of scores, for each track of rows
  static constexpr int kRows = WIDE ? 256 : 128;  // of a block
  static constexpr int kShared = WIDE ? 1 : 128;  // rows that two threads share
  static constexpr int kProducers = 4;            // warps
  static constexpr int kThreads = 512;
  static constexpr int kEntry = kKeys * D * 2;
  // queries of two segments where there is room, so that the next one's are there in time
  static constexpr int kQs = WIDE || D == 256 ? 1 : 2;
  static constexpr int kEntries = D == 64 ? (WIDE ? 8 : 6) : E8 ? 3 : 4;
  static constexpr int kStages = !E8 ? 0 : D == 64 ? 4 : 3;  // entries of codes on their way
  static constexpr int kScales = !E8 ? 0 : D == 128 ? 3 : 8;  // tiles whose columns' scales are kept, from their codes' copies to the softmax
  // two producer warps for keys and two for values, where each kind has its own places (an odd number
  // of them passes from one kind to the other, and a wait for the one would not see the other's turn)
  static constexpr bool kSplit = kEntries % 2 == 0 && kStages % 2 == 0 && !(E8 && WIDE);
  static constexpr int kBring = kSplit ? kProducers / 2 : kProducers;  // warps that bring an entry
  static constexpr int kTurn = 2;  // tiles that a segment's end is worth in the dealing (it takes 6-9 k clk)
  static constexpr int kQBytes = kRows * D * 2;
  static constexpr int kNeed = kQs * kQBytes + kEntries * kEntry + kStages * kEntry / 2;
  static constexpr int kSmem = kNeed > kPdlTmemSmem ? kNeed : kPdlTmemSmem + 1024;
  static constexpr int kCols = WIDE ? kKeys : kKeys / 2;  // columns of a thread
  // TMEM columns
  static constexpr int kO = 0, kOStep = 128, kS = 256, kSStep = kKeys;
  // weights take the place of their scores: of kGroup keys a thread at a time, the high parts, then the low ones
  static constexpr int kGroup = kCols >= 64 ? 64 : 32;
  static_assert(kSmem > kPdlTmemSmem, "no second kernel with tensor memory beside it");
};

struct Info {  // a tile
  uint32_t valid[4];  // its positions that exist: in the sequence's range, on present pages
  int p0, n, lo, flags;  // first position; the sequence's length and lowest position; 1: rows attend to it differently (segment from bit 1 on)
  // 8 bits: whether columns have scales of their own; else 2^E of the keys (their rows' factor taken out), E of the values
  int key_columns, value_columns;
  float ek, ev;
};

template <class S>
struct Control {
  uint64_t full[8], empty[8], info[kInfos], paged[8], placed[4], taken[4], staged[4], unstaged[4], q_full[2], q_empty[2], s_full[4], p_full[4], pv_done[2], used[8], fin;
  Info tile[kInfos];
  unsigned long long bad[16][2];  // per segment: nodes, and positions from lo on, with values that are not finite
  int64_t off[4][S::kKeys];      // element offsets of a tile's rows, -1: none
  int page[8][S::kKeys];         // pages of a tile's rows, -1: none
  uint8_t fac[4][2][S::kScales ? S::kKeys : 1];  // 2^(e - E) of each row of an 8-bit tile in fp16, its upper byte; 1 with scales by column
  // of each position of an 8-bit tile: key scale, exponent of the value scale, and 2 to minus that
  float4 scale[S::kScales ? S::kScales : 1][3][S::kScales ? S::kKeys / 4 : 1];
  union {
    int64_t sum[16];       // of the warps' tiles, at the start
    float qf[3][S::kRows];  // what is left of a query's scale
  };
  float mx[2][2][S::kShared];  // maxima (a segment's sums at its end)
  long long patience;  // of a wait, in clocks
  int where[5];  // sequence, key head and block, tile, length; what the share has of a segment's end ahead of that
  uint32_t tmem;
  int err;
};

// Division of x < 2^31 by d with a product: with 2^s the power of two at or above d,
// m = floor(2^(31 + s) / d) + 1 (Granlund and Montgomery); m = 0: a shift alone
struct Divisor {
  uint32_t m, s;
  __device__ __forceinline__ int of(int x) const { return (int)((m ? __umulhi((uint32_t)x, m) : (uint32_t)x) >> s); }
};
static inline Divisor divisor(uint32_t d) {
  Divisor r{0, 0};
  while ((1u << r.s) < d) ++r.s;
  if ((1u << r.s) != d) r.m = (uint32_t)(((uint64_t)1 << (31 + r.s)) / d + 1), --r.s;
  return r;
}

struct Args {
  TreeArgs a;
  int groups, blocks;             // groups: key heads x blocks of rows
  Divisor page, group;            // by the page size, by the query heads of a key head
  float* part;
  SegMeta* meta;
  int32_t* error;
  long long patience;  // clocks after which a wait gives up
  bool hold;           // self-test: no tile is placed, every wait for one runs out
};

struct Seg {
  int b, hk, blk, nt, n, lo, end, base;  // sequence, key head, block of rows; tiles; ...
};

template <int KEYS>
__device__ __forceinline__ void seg_range(const TreeArgs& a, int len, Seg& s) {
  const int cap = a.c.max_pages * a.c.page_size;
  s.n = min(max(len, 0), cap);
  s.lo = a.window > 0 ? max(0, s.n + (a.mask ? 1 : 0) - a.window) : 0;
  s.end = a.mask ? min(cap, s.n + a.n_nodes) : s.n;
  s.base = s.lo & ~(KEYS - 1);
  s.nt = max(1, (s.end - s.base + KEYS - 1) / KEYS);  // an empty sequence has one empty tile
}

// The line of `total` tiles dealt out to `workers` CTAs: the first `more` get one
// more than the others.
__device__ __forceinline__ int64_t quotient(int64_t a, int b) {  // of numbers that mostly have 32 bits
  return a >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}
struct Deal {
  int64_t each;
  int more;
  __device__ __forceinline__ Deal(int64_t total, int workers) : each(quotient(total, workers)), more((int)(total - each * workers)) {}
  __device__ __forceinline__ int64_t start(int w) const { return w * each + min(w, more); }
  __device__ __forceinline__ int worker(int64_t tile) const {
    const int64_t cut = more * (each + 1);
    return each >> 30 ? (tile < cut ? (int)(tile / (each + 1)) : more + (int)((tile - cut) / each))
                      : (tile < cut ? (int)quotient(tile, (int)each + 1) : more + (int)quotient(tile - cut, (int)each));
  }
};

// the CTA's share of the line, segment by segment; every role walks it
template <int KEYS, int TURN>
struct Walk {
  const Args& g;
  Seg s;
  int ct, cnt, ahead, index;  // first tile and tiles of this CTA in the segment; the next sequence's length; segments behind
  int64_t left;               // of the share, this segment's part included
  __device__ __forceinline__ Walk(const Args& g, const int* where, int64_t share) : g(g) {
    s.b = where[0], s.hk = where[1] / g.blocks, s.blk = where[1] % g.blocks, ct = where[2], index = 0;
    seg_range<KEYS>(g.a, where[3], s);
    ahead = g.a.lens[min(s.b + 1, g.a.c.n_seqs - 1)];
    left = share;
    cnt = (int)min((int64_t)(s.nt - ct), left);
  }
  __device__ __forceinline__ bool next() {
    left -= s.nt + TURN - ct;
    if (left <= 0) return false;
    ct = 0;
    ++index;
    advance();
    cnt = (int)min((int64_t)s.nt, left);
    return true;
  }
  __device__ __forceinline__ void advance() {
    if (++s.blk < g.blocks) return;
    s.blk = 0;
    if (++s.hk < g.a.c.n_heads) return;
    s.hk = 0;
    ++s.b;
    seg_range<KEYS>(g.a, ahead, s);
    ahead = g.a.lens[min(s.b + 1, g.a.c.n_seqs - 1)];
  }
};

// ---------------------------------------------------------------- PTX
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// A whole warp runs the role that issues products, so that what goes into them stays in
// uniform registers; one lane, the leader, issues.  (One lane in a branch of its own took 65 clk for
// each instruction, what the tensor core takes for 128 x 128 x 16.)
__device__ __forceinline__ bool elect() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0;
}
__device__ __forceinline__ uint64_t desc_of(uint32_t lo, uint32_t hi) { return (uint64_t)hi << 32 | lo; }
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t leader) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t"
      "}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(leader));
}
// A (16-bit, K-major) from TMEM
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t leader) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t"
      "}\n" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(leader));
}
template <typename T> constexpr uint32_t idesc(int M, int N, int b_mn) {
  const uint32_t fmt = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
  return (1u << 4) | (fmt << 7) | (fmt << 10) | ((uint32_t)b_mn << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// 32 columns of the thread's lane, without waiting
__device__ __forceinline__ void ld32(uint32_t at, float (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
      "%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
        "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]),
        "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]),
        "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(at));
}
__device__ __forceinline__ void ld_wait(float (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]),
                 "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]), "+f"(v[17]),
                 "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]),
                 "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
               :
               : "memory");
}
__device__ __forceinline__ void st16(uint32_t at, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at), "r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
      "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ bool mbar_test(uint64_t* b, uint32_t parity) {  // without suspending
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t"
      "}\n"
      : "=r"(ok)
      : "r"(tc::smem_u32(b)), "r"(parity)
      : "memory");
  return ok != 0;
}

// A bounded wait; once one has given up, the others do not wait either.  The roles then run through what is
// left of their share without waiting (the warps of a named barrier stay in step), over whatever shared memory
// holds: what addresses come from is either as it was set at the start, nothing there, or of some tile of the
// share, and page numbers are held against n_pages where they are used.  The results are not; the flag says so.
__device__ __forceinline__ void wait_long(int* err, long long patience, uint64_t* b, uint32_t parity) {
  const long long t0 = clock64();
  while (!tc::mbar_try_wait(b, parity)) {
    if (*(volatile int*)err) return;
    if (clock64() - t0 > patience) {
      atomicExch(err, 1);
      return;
    }
  }
}
template <class C>
__device__ __forceinline__ void wait(C& c, uint64_t* b, uint32_t parity) {
  if (__builtin_expect(!tc::mbar_try_wait(b, parity), 0)) wait_long(&c.err, c.patience, b, parity);
}

// the weight of a piece with maximum m where the largest is mm; a piece that
// met nothing has m = -inf, sum 0
__device__ __forceinline__ float piece_weight(float m, float mm) {
  return m == -CUDART_INF_F ? (mm == -CUDART_INF_F ? 1.0f : 0.0f) : exp2_fast(m - mm);
}

// fp16 weights are e^(s - m) 2^kBias, at most 2^(kBias + kLag): what is 2^-30 of the largest is kept
// (8 bits: 2^-27 of the largest weight times scale, for a tile's E counts for up to 5 more than a row's exponent)
template <typename M, bool E8> struct Weights;
template <> struct Weights<__nv_bfloat16, false> {
  static constexpr float kBias = 0.0f, kLag = 8.0f;
};
template <> struct Weights<__half, false> {
  static constexpr float kBias = 6.0f, kLag = 8.0f;
};
template <> struct Weights<__half, true> {
  static constexpr float kBias = 7.0f, kLag = 8.0f;
};
template <typename M, bool E8> __device__ __forceinline__ float log_sum(float m, float l) {
  return l == 0.0f ? -CUDART_INF_F : (m == -CUDART_INF_F ? 0.0f : m - Weights<M, E8>::kBias) * 0.69314718f + logf(l);
}

// the first 16-bit part of two weights, packed, and what it leaves of them
template <typename M> __device__ __forceinline__ float2 high_part(float2 p, uint32_t& high) {
  high = pack2<M>(p.x, p.y);
  const float2 h = unpack2<M>(high);
  return make_float2(p.x - h.x, p.y - h.y);
}

template <typename M> __device__ __forceinline__ bool not_finite(uint32_t w, int half) {
  const uint32_t e = std::is_same<M, __nv_bfloat16>::value ? 0x7f80u : 0x7c00u;
  return ((w >> (16 * half)) & e) == e;
}

// byte address of 16-byte chunk ch of row r in a swizzled tile of `rows` rows
__device__ __forceinline__ uint32_t chunk_at(int r, int ch, int rows) {
  return (ch >> 3) * rows * 128 + r * 128 + (((ch & 7) ^ (r & 7)) << 4);
}

// which of elements d .. d + 15 of the marked positions' values (nodes, positions from lo on) are not finite
template <typename T, bool E8>
__device__ __noinline__ uint32_t spoilt_columns(const TreeArgs& a, int b, int hk, int n, int lo, uint64_t nodes, uint64_t ahead, int d) {
  const pe_kv_cache& c = a.c;
  uint32_t nan = 0;
#pragma unroll 1
  for (int k = 0; k < 128; ++k) {
    if (!((k < 64 ? nodes >> k : ahead >> (k - 64)) & 1)) continue;
    const int p = k < 64 ? n + k : lo + k - 64;
    if (p >= c.max_pages * c.page_size) continue;
    const int page = c.table[(int64_t)b * c.table_stride + p / c.page_size], sl = p % c.page_size;
    if (page < 0 || page >= c.n_pages) continue;  // (marks after a wait that gave up may be another segment's)
    const int64_t at = kv_page_offset(c, page) + (int64_t)sl * c.slot_stride + hk * c.head_stride + d;
#pragma unroll 1
    for (int j = 0; j < 16; ++j)
      if (E8 ? (((const uint8_t*)c.v)[at + j] & 0x7f) == 0x7f : not_finite<T>(((const uint16_t*)c.v)[at + j], 0)) nan |= 1u << j;
  }
  return nan;
}

// What is not the same for every column and row, in functions apart from the kernel's body, whose roles' code the
// instruction cache has to hold.

// Scores of `COLS` columns from `first` of tile f on, in their place: -inf where the row does not attend; over 8
// bits in powers of two, columns' own scales and their values' exponents in them
template <bool E8, int COLS, int KEYS>
__device__ __noinline__ void set_apart(uint32_t sc, const Info& f, int first, int row_lo, uint64_t bits, bool live, const float4* scale, float cs) {
  const bool keys = E8 && f.key_columns, values = E8 && f.value_columns;
#pragma unroll 1
  for (int i = 0; i < COLS / 32; ++i) {
    const int pw = f.p0 + first + 32 * i;
    const int below = min(max(f.n - pw, 0), 32), skip = min(max(row_lo - pw, 0), 32);
    uint32_t ctx = below == 32 ? 0xffffffffu : (1u << below) - 1;
    ctx &= skip == 32 ? 0u : 0xffffffffu << skip;
    const int sh = pw - f.n;
    const uint32_t nodes = sh >= 64 || sh <= -32 ? 0u : sh >= 0 ? (uint32_t)(bits >> sh) : (uint32_t)(bits << -sh);
    const uint32_t kept = live ? f.valid[(first >> 5) + i] & (ctx | nodes) : 0u;
    float x[32];
    ld32(sc + 32 * i, x);
    ld_wait(x);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t r[16];
#pragma unroll
      for (int j = 0; j < 16; j += 4) {
        float4 k = make_float4(1.0f, 1.0f, 1.0f, 1.0f), e = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (keys) k = scale[8 * i + 4 * h + j / 4];
        if (values) e = scale[KEYS / 4 + 8 * i + 4 * h + j / 4];
        float z[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) z[u] = x[16 * h + j + u];
        if (E8) z[0] = fmaf(z[0] * k.x, cs, e.x), z[1] = fmaf(z[1] * k.y, cs, e.y), z[2] = fmaf(z[2] * k.z, cs, e.z), z[3] = fmaf(z[3] * k.w, cs, e.w);
#pragma unroll
        for (int u = 0; u < 4; ++u) r[j + u] = __float_as_uint((kept >> (16 * h + j + u)) & 1 ? z[u] : -CUDART_INF_F);
      }
      st16(sc + 32 * i + 16 * h, r);
    }
  }
  st_wait();
}
// an output whose weights' reference has moved
__device__ __forceinline__ void rescale(uint32_t at, int columns, float f) {
#pragma unroll 1
  for (int i = 0; i < columns; i += 16) {
    float o[16];
    tc::tmem_ld16(at + i, o);
    uint32_t r[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) r[j] = __float_as_uint(o[j] * f);
    st16(at + i, r);
  }
}

// bit of row r's values, if rows attend to them differently: of a node (which 0), of a position from lo on (1)
__device__ __forceinline__ uint64_t apart_bit(const Info& f, int r, int window, int n_nodes, int& which) {
  const int p = f.p0 + r, node = p - f.n;
  which = 0;
  if (node >= 0) return node < n_nodes ? 1ull << node : 0;
  which = 1;
  return window > 0 && p >= f.lo && p - f.lo < 64 ? 1ull << (p - f.lo) : 0;
}
// Values that are not finite, where rows attend to them differently, become zeros and a mark: a thread's chunks of a tile
template <typename T, int KEYS, int PASS>
__device__ __noinline__ void clean_values(unsigned char* entry, const Info& f, unsigned long long* bad, int window, int n_nodes, int row0, int ch) {
  // (nodes' rows alone, where there is no window)
  const int from = window > 0 ? 0 : max(f.n - f.p0, 0), to = window > 0 ? KEYS : min(KEYS, f.n + n_nodes - f.p0);
#pragma unroll 1
  for (int r = row0 + (from - row0 + PASS - 1) / PASS * PASS; r < to; r += PASS) {
    if (r < from) continue;
    int which;
    const uint64_t bit = apart_bit(f, r, window, n_nodes, which);
    if (!bit || !((f.valid[r >> 5] >> (r & 31)) & 1)) continue;
    uint4* p = reinterpret_cast<uint4*>(entry + chunk_at(r, ch, KEYS));
    uint4 x = *p;
    uint32_t* y = reinterpret_cast<uint32_t*>(&x);
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (not_finite<T>(y[i], 0)) y[i] &= 0xffff0000u, any = true;
      if (not_finite<T>(y[i], 1)) y[i] &= 0x0000ffffu, any = true;
    }
    if (any) {
      *p = x;
      atomicOr(&bad[which], bit);
    }
  }
}
// The same of codes that are no numbers, in their stage (a scale that is none is in its column of scores, masked like those)
template <int EACH, int PASS, int THREADS>
__device__ __noinline__ void clean_codes(unsigned char* from, const Info& f, unsigned long long* bad, int window, int n_nodes, int row0) {
#pragma unroll 1
  for (int i = 0; i < EACH; ++i) {
    const int r = row0 + i * PASS;
    if (window == 0 && (i + 1) * PASS <= f.n - f.p0) continue;  // no nodes there
    int which;
    const uint64_t bit = (f.valid[r >> 5] >> (r & 31)) & 1 ? apart_bit(f, r, window, n_nodes, which) : 0;
    if (!bit) continue;
    uint4 z = *reinterpret_cast<const uint4*>(from + i * THREADS * 16);
    uint32_t* y = reinterpret_cast<uint32_t*>(&z);
    bool any = false;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int b = 0; b < 32; b += 8)
        if (((y[j] >> b) & 0x7f) == 0x7f) y[j] &= ~(0xffu << b), any = true;
    if (any) {
      *reinterpret_cast<uint4*>(from + i * THREADS * 16) = z;
      atomicOr(&bad[which], bit);
    }
  }
}

// a lane's bytes as what those take, 32 positions apart (what is not there is masked: any number will do)
static __device__ __noinline__ void column_scales(float* to, bool values, int keys, int b0, int b1, int b2, int b3) {
#pragma unroll 1
  for (int r = 0; r < keys; r += 32) {
    const int e = min(max(b0, 63), 247);
    to[r] = b0 < 0 ? 0.0f : !values ? key_scale(b0) : b0 == 255 ? CUDART_NAN_F : (float)(e - 127);
    if (values) to[keys + r] = __int_as_float((254 - e) << 23);
    b0 = b1, b1 = b2, b2 = b3;
  }
}
// l and the sum of those columns' weights with the value scales taken out
template <int COLS, int KEYS>
__device__ __noinline__ float column_sum(uint32_t sc, const float4* scale, float off, float l) {
#pragma unroll 1
  for (int i = 0; i < COLS / 32; ++i) {
    float x[32];
    ld32(sc + 32 * i, x);
    ld_wait(x);
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
      const float4 back = scale[2 * (KEYS / 4) + 8 * i + j / 4];
      l = fmaf(exp2_fast(x[j] + off), back.x, l);
      l = fmaf(exp2_fast(x[j + 1] + off), back.y, l);
      l = fmaf(exp2_fast(x[j + 2] + off), back.z, l);
      l = fmaf(exp2_fast(x[j + 3] + off), back.w, l);
    }
  }
  return l;
}

// ---------------------------------------------------------------- the kernel
// T: type of queries and output; E8: an 8-bit cache
template <typename T, bool E8, int D, bool WIDE>
__global__ void __launch_bounds__(Shape<D, E8, WIDE>::kThreads, 1) attn_kernel(Args g) {
  using S = Shape<D, E8, WIDE>;
  using M = typename std::conditional<E8, __half, T>::type;  // type of the products
  constexpr int kKeys = S::kKeys, kChunks = D / 8, kEntries = S::kEntries, kTurn = S::kTurn;
  constexpr bool kLow = !std::is_same<M, __half>::value || std::is_same<T, __half>::value;  // weights have a low part
  extern __shared__ __align__(1024) unsigned char smem[];  // (a swizzle's atoms)
  __shared__ __align__(16) Control<S> ctl;
  static_assert(S::kSmem + (sizeof(Control<S>) + 1023) / 1024 * 1024 <= 232448, "shared memory of an SM");
  const TreeArgs& a = g.a;
  const pe_kv_cache& c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t qs = tc::smem_u32(smem), ring = qs + S::kQs * S::kQBytes;
  const int G = a.n_q_heads / c.n_heads, R = a.n_nodes * G, B = c.n_seqs;

  if (qs & 1023) {  // a base that is not what it was declared to be
    if (tid == 0) atomicExch(g.error, 1);
    return;
  }
  if (warp == 8) tc::tmem_alloc(&ctl.tmem, 512);
  if (tid == 0) {
    for (int i = 0; i < 8; ++i) {
      tc::mbar_init(&ctl.full[i], E8 ? S::kBring : 32 * S::kBring);
      tc::mbar_init(&ctl.empty[i], 1);
    }
    constexpr int kPlacers = E8 ? 3 : 1;  // warps: places, scales of keys, of values
    for (int i = 0; i < kInfos; ++i) tc::mbar_init(&ctl.info[i], kPlacers);
    for (int i = 0; i < 8; ++i) tc::mbar_init(&ctl.used[i], 8);
    for (int i = 0; i < 8; ++i) tc::mbar_init(&ctl.paged[i], 1);
    for (int i = 0; i < 4; ++i) {
      tc::mbar_init(&ctl.placed[i], kPlacers);
      tc::mbar_init(&ctl.taken[i], E8 ? S::kProducers + 2 : S::kProducers);
      tc::mbar_init(&ctl.s_full[i], 1);
      tc::mbar_init(&ctl.p_full[i], WIDE ? 4 : 8);
      tc::mbar_init(&ctl.staged[i], 32);
      tc::mbar_init(&ctl.unstaged[i], S::kBring);
    }
    tc::mbar_init(&ctl.fin, 1);
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(&ctl.q_full[i], E8 ? S::kBring : 32);
      tc::mbar_init(&ctl.q_empty[i], 1);
      tc::mbar_init(&ctl.pv_done[i], 1);
    }
    ctl.err = 0;
    ctl.patience = g.patience;
    tc::fence_mbar_init();
  }
  // nothing is there: what a role finds whose wait for a tile gave up
  for (int i = tid; i < 4 * kKeys; i += S::kThreads) (&ctl.off[0][0])[i] = -1;
  for (int i = tid; i < 8 * kKeys; i += S::kThreads) (&ctl.page[0][0])[i] = -1;
  if (tid < kInfos) ctl.tile[tid] = Info{}, ctl.bad[tid][0] = ctl.bad[tid][1] = 0;
  cudaGridDependencySynchronize();
  cudaTriggerProgrammaticLaunchCompletion();

  // -- a prefix sum of the sequences' tiles finds where this CTA's share starts
  const int chunk = (B + S::kThreads - 1) / S::kThreads;
  int64_t sum = 0;
  Seg s0;
  for (int b = tid * chunk; b < min(B, (tid + 1) * chunk); ++b) {
    seg_range<kKeys>(a, a.lens[b], s0);
    sum += s0.nt + kTurn;
  }
  int64_t incl = sum;
  for (int x = 1; x < 32; x <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, incl, x);
    if (lane >= x) incl += y;
  }
  if (lane == 31) ctl.sum[warp] = incl;
  tc::fence_before();
  __syncthreads();
  tc::fence_after();
  int64_t before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < S::kThreads / 32; ++w) {
    if (w < warp) before += ctl.sum[w];
    total += ctl.sum[w];
  }
  total *= g.groups;
  const int workers = (int)min(total, (int64_t)gridDim.x);
  const Deal deal(total, workers);
  const int64_t start = (int)blockIdx.x < workers ? deal.start(blockIdx.x) : 0;
  int64_t share = (int)blockIdx.x < workers ? deal.start(blockIdx.x + 1) - start : 0;
  const int64_t lo = (before + incl - sum) * g.groups, hi = (before + incl) * g.groups;
  if (start >= lo && start < hi) {
    int64_t at = lo;
    int b = tid * chunk, len = 0;
    for (;; ++b) {
      len = a.lens[b];
      seg_range<kKeys>(a, len, s0);
      if (start < at + (int64_t)(s0.nt + kTurn) * g.groups) break;
      at += (int64_t)(s0.nt + kTurn) * g.groups;
    }
    int grp = (int)quotient(start - at, s0.nt + kTurn), skip = 0;
    int ct = (int)(start - at - (int64_t)grp * (s0.nt + kTurn));
    if (ct >= s0.nt) {
      // the share starts within a segment's end: with the next segment, if it has one
      skip = s0.nt + kTurn - ct;
      ct = 0;
      if (++grp == g.groups) {
        grp = 0;
        if (++b < B) len = a.lens[b];
      }
    }
    ctl.where[0] = b, ctl.where[1] = grp, ctl.where[2] = ct, ctl.where[3] = len, ctl.where[4] = skip;
    SegMeta m{0, 0, 0, 0};
    if (share > skip && ct > 0) {
      // the boundary at this CTA's start joins the segment if it is the first inside it
      const int64_t g0 = start - ct, prev = deal.start((int)blockIdx.x - 1);
      if (prev <= g0) {
        m.seq = b, m.group = grp;
        m.pieces = deal.worker(g0 + s0.nt - 1) - blockIdx.x + 2;
        m.first_slot = 2 * (blockIdx.x - 1) + (prev < g0 - kTurn ? 1 : 0);  // (not its first segment)
      }
    }
    if (share > 0) g.meta[blockIdx.x] = m;
  }
  if (tid == 0 && share <= 0) g.meta[blockIdx.x] = SegMeta{0, 0, 0, 0};
  __syncthreads();
  const uint32_t tmem = ctl.tmem;
  share -= share > 0 ? ctl.where[4] : 0;

  if (share <= 0) {
    // nothing to do
  } else if (warp < 8) {
    // ================================================== softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 160;");  // 256 threads of 160 and 256 of 96: what 512 of 128 had
    const int wg = warp >> 2, row = (warp & 3) * 32 + lane;  // row of the tile, lane of TMEM
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const float qlog = fabsf(a.scale) * 1.4426950408889634f;
    uint32_t sp[2] = {0, 0}, pp = 0, ip = 0;  // phases: scores, outputs, tiles seen
    uint64_t bits = 0;  // the row's mask, of sequence last_b
    int last_b = -1;
    Walk<kKeys, kTurn> w(g, ctl.where, share);
    do {
      const Seg& s = w.s;
      const int hk = s.hk, r0 = s.blk * S::kRows, rows = min(R - r0, S::kRows);
      const int rr = r0 + (WIDE ? wg * 128 : 0) + row;  // row of the sequence and key head
      const bool exists = rr < R && (WIDE ? wg * 128 + row < rows : row < rows);
      const int node = exists ? g.group.of(rr) : 0, head = hk * G + (exists ? rr - node * G : 0);
      int row_lo = s.lo;
      bool live = exists;
      if (a.mask) {
        if (s.b != last_b || g.blocks > 1) bits = exists ? a.mask[s.b * a.mask_stride + node] & (0xffffffffffffffffull >> (64 - a.n_nodes)) : 0;
        last_b = s.b;
        live = bits != 0;
        if (a.window > 0) row_lo = max(0, s.n + __popcll(bits) - a.window);
      }
      const int lo_hi = a.mask && a.window > 0 ? max(0, s.n + 64 - a.window) : s.lo;
      const bool warp_live = __any_sync(0xffffffffu, exists);
      const bool both = !WIDE || rows > 128;  // the second warpgroup has work
      float m = -CUDART_INF_F, l = 0.0f, qf = 1.0f;
      auto use = [&](uint32_t tile) {  // the warp has read the tile's scales
        __syncwarp();
        if (E8 && lane == 0) tc::mbar_arrive(&ctl.used[tile & 7]);
      };
      if (WIDE && wg == 1 && !both) {
        if constexpr (E8)
          for (int t = 0; t < w.cnt; ++t, ++ip) {
            wait(ctl, &ctl.info[ip % kInfos], (ip / kInfos) & 1);
            use(ip);
          }
        else
          ip += w.cnt;
        continue;
      }
      for (int t = 0; t < w.cnt; ++t, ++ip) {
        const int b2 = t % S::kBufs, buf = WIDE ? wg : b2;  // of scores and weights
        // (passed too early by a warpgroup that left 16 tiles out: then the scores' barrier is what holds it)
        wait(ctl, &ctl.info[ip % kInfos], (ip / kInfos) & 1);
        const Info& f = ctl.tile[ip % kInfos];
        wait(ctl, &ctl.s_full[buf], sp[b2] & 1);
        ++sp[b2];
        __syncwarp();
        tc::fence_after();
        if (E8 && t == 0) qf = ctl.qf[w.index % 3][(WIDE ? wg * 128 : 0) + row];
        const bool kcol = E8 && f.key_columns, vcol = E8 && f.value_columns;
        const float ev = E8 ? f.ev : 0.0f;
        const bool whole = f.p0 >= lo_hi && f.p0 + kKeys <= f.n && (f.valid[0] & f.valid[1] & f.valid[2] & f.valid[3]) == 0xffffffffu;
        const bool apart = !whole || kcol || vcol;
        // what takes a score to powers of two (a scale of 0 as the least there is, what is masked stays -inf)
        const float cs = E8 ? qlog * (qf * f.ek) : qlog, cf = E8 && apart ? 1.0f : fmaxf(cs, 1e-37f);
        const float2 cf2 = make_float2(cf, cf);
        const float4* scale = &ctl.scale[E8 ? ip % (E8 ? S::kScales : 1) : 0][0][E8 && !WIDE ? wg * (S::kCols / 4) : 0];
        if (warp_live) {
          const uint32_t sc = lanes + S::kS + buf * S::kSStep + (WIDE ? 0 : wg * S::kCols);
          // 64 columns at a time (head_dim 256: 32); code is kept short, for the roles share the instruction cache
          constexpr int kHalves = S::kCols >= 64 ? 2 : 1, kTurns = S::kCols / (32 * kHalves);
          if (__builtin_expect(apart, 0)) set_apart<E8, S::kCols, kKeys>(sc, f, WIDE ? 0 : wg * S::kCols, row_lo, bits, live, scale, cs);
          float v[kHalves][32];
          auto fetch = [&](int turn) {
#pragma unroll
            for (int h = 0; h < kHalves; ++h) ld32(sc + 64 * turn + 32 * h, v[h]);
#pragma unroll
            for (int h = 0; h < kHalves; ++h) ld_wait(v[h]);
          };
          // the row's largest score
          float top = -CUDART_INF_F;
#pragma unroll 1
          for (int turn = 0; turn < kTurns; ++turn) {
            fetch(turn);
            float most[4] = {top, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
#pragma unroll
              for (int j = 0; j < 32; j += 8)
#pragma unroll
                for (int i = 0; i < 4; ++i) most[i] = fmaxf(most[i], fmaxf(v[h][j + 2 * i], v[h][j + 2 * i + 1]));
            top = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
          }
          if (!WIDE) {
            ctl.mx[ip & 1][wg][row] = top;
            bar_sync(1 + (warp & 3), 64);
            top = fmaxf(top, ctl.mx[ip & 1][wg ^ 1][row]);
          }
          top = top == -CUDART_INF_F ? top : fmaf(top, cf, ev);
          const bool over = top > m + Weights<M, E8>::kLag;
          if (__builtin_expect(__any_sync(0xffffffffu, over), 0)) {
            const float x = over ? top : m;
            const float fr = over ? (m == -CUDART_INF_F ? 0.0f : exp2_fast(m - x)) : 1.0f;
            m = x;
            l *= fr;
            if (t > 0) {
              wait(ctl, &ctl.pv_done[WIDE ? wg : 0], (pp - 1) & 1);  // the last product into the output
              __syncwarp();
              tc::fence_after();
              rescale(lanes + S::kO + (WIDE ? wg * S::kOStep : wg * (D / 2)), WIDE ? D : D / 2, fr);
            }
          }
          const float off = ev + Weights<M, E8>::kBias - (m == -CUDART_INF_F ? 0.0f : m);
          const float2 off2 = make_float2(off, off);
          float2 part = make_float2(0.0f, 0.0f);
          if (E8 && __builtin_expect(vcol, 0)) l = column_sum<S::kCols, kKeys>(sc, scale, off, l);
#pragma unroll 1
          for (int turn = 0; turn < kTurns; ++turn) {
            if (kTurns > 1) fetch(turn);
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
              uint32_t pk[16], low[kLow ? 16 : 1];
#pragma unroll
              for (int j = 0; j < 32; j += 2) {
                const float2 e = __ffma2_rn(make_float2(v[h][j], v[h][j + 1]), cf2, off2);
                const float2 p = make_float2(exp2_fast(e.x), exp2_fast(e.y));
                part = __fadd2_rn(part, p);
                if constexpr (kLow) {
                  const float2 rest = high_part<M>(p, pk[j / 2]);
                  low[j / 2] = pack2<M>(rest.x, rest.y);
                } else {
                  pk[j / 2] = pack2<M>(p.x, p.y);
                }
              }
              st16(sc + 64 * turn + 16 * h, pk);
              if constexpr (kLow) st16(sc + 64 * turn + S::kGroup / 2 + 16 * h, low);
            }
          }
          if (!vcol) l = E8 ? fmaf(part.x + part.y, exp2f(-ev), l) : l + (part.x + part.y);
          st_wait();
        } else if (!WIDE) {
          bar_sync(1 + (warp & 3), 64);
        }
        if (E8) use(ip);
        // The end waits for the last output, so the one before it has to be seen first (scores say that all
        // but two are done), and while the last one cannot be: a barrier two phases on looks like none
        if (t > 0 && t == w.cnt - 1) wait(ctl, &ctl.pv_done[WIDE ? wg : 0], (pp - 1) & 1);
        tc::fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&ctl.p_full[buf]);
        ++pp;
      }
      // -- the segment, or this CTA's part of it, ends
      wait(ctl, &ctl.pv_done[WIDE ? wg : 0], (pp - 1) & 1);
      __syncwarp();
      tc::fence_after();
      if (!live) m = -CUDART_INF_F, l = 0.0f;
      if (!WIDE) {
        // (in place of the last tile's maxima: all have read those, or its output would not be there)
        float (&sums)[2][S::kShared] = ctl.mx[(ip - 1) & 1];
        sums[wg][row] = l;
        bar_sync(1 + (warp & 3), 64);
        l += sums[wg ^ 1][row];
      }
      if (warp_live) {
        const bool whole = w.ct == 0 && w.cnt == s.nt;
        const uint64_t bad_node = ctl.bad[w.index & 15][0] & bits;
        uint64_t bad_pos = ctl.bad[w.index & 15][1];
        if (row_lo > s.lo) bad_pos &= row_lo - s.lo >= 64 ? 0 : 0xffffffffffffffffull << (row_lo - s.lo);
        const bool spoilt = live && (bad_node | bad_pos) != 0;
        constexpr int kMine = WIDE ? D : D / 2;  // elements of the thread
        const int d0 = WIDE ? 0 : wg * kMine;
        const uint32_t oc = lanes + S::kO + (WIDE ? wg * S::kOStep : d0);
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        T* out = (T*)a.out + s.b * a.o_seq + node * a.o_node + head * a.o_head + d0;
        // a CTA has two slots: its first segment's, and that of a segment it starts and does not end
        const int64_t slot = 2 * (int64_t)blockIdx.x + (w.index > 0 ? 1 : 0);
        float* piece = g.part + slot * S::kRows * (D + 2);
        const int prow = (WIDE ? wg * 128 : 0) + row;
        float* to = piece + (int64_t)prow * D + d0;
        // short code again: it is fetched anew for each segment (with the parts of a row spread over lanes, for
        // stores of 128 bytes, it took twice as long)
#pragma unroll 1
        for (int i = 0; i < kMine; i += 16) {
          float v[16];
          tc::tmem_ld16(oc + i, v);
          if (__builtin_expect(spoilt, 0)) {  // an attended value that is not finite makes its element NaN
            const uint32_t nan = spoilt_columns<T, E8>(a, s.b, hk, s.n, s.lo, bad_node, bad_pos, d0 + i);
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if ((nan >> j) & 1) v[j] = CUDART_NAN_F;
          }
          if (l == 0.0f)  // nothing attended to, whatever the values are
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = 0.0f;
          if (exists && whole) {
#pragma unroll
            for (int j = 0; j < 16; j += 8)
              *reinterpret_cast<uint4*>(out + i + j) = make_uint4(pack2<T>(v[j] * inv, v[j + 1] * inv), pack2<T>(v[j + 2] * inv, v[j + 3] * inv),
                                                                  pack2<T>(v[j + 4] * inv, v[j + 5] * inv), pack2<T>(v[j + 6] * inv, v[j + 7] * inv));
          } else if (exists) {
#pragma unroll
            for (int j = 0; j < 16; j += 4) *reinterpret_cast<float4*>(to + i + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
          }
          __syncwarp();
        }
        if (exists && (WIDE || wg == 0)) {
          if (whole) {
            if (a.lse) a.lse[((int64_t)s.b * a.n_nodes + node) * a.n_q_heads + head] = log_sum<M, E8>(m, l);
          } else {
            piece[S::kRows * D + prow] = m;
            piece[S::kRows * (D + 1) + prow] = l;
          }
        }
      }
      tc::fence_before();
    } while (w.next());
  } else if (warp < 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
    constexpr int kPlace = E8 ? 1 : 2;  // warps that place, every kPlace-th tile each
    if (warp >= 9 && warp < 9 + kPlace && !g.hold) {
    // ================================================== places
      // A lane finds the places of rows lane, lane + 32, ...; table entries are copied kAhead turns ahead
      constexpr int kMine = kKeys / 32, kAhead = 3;
      Walk<kKeys, kTurn> nx(g, ctl.where, share);
      int nt = 0;
      auto on = [&](Walk<kKeys, kTurn>& w, int& t, int n) {  // n tiles on; false past the end
        bool there = true;
        for (; n > 0 && there; --n)
          if (++t == w.cnt) {
            t = 0;
            there = w.next();
          }
        return there;
      };
      bool more = on(nx, nt, warp - 9), here = more;
      Walk<kKeys, kTurn> far = nx;
      int tf = nt;
#pragma unroll 1
      for (int64_t at = warp - 9 - kAhead * kPlace; here; at += kPlace) {
        if (more) {  // table entries of tile at + kAhead * kPlace
          const int p0 = far.s.base + (far.ct + tf) * kKeys;
          int* to = ctl.page[(uint32_t)(at + kAhead * kPlace) & 7];
#pragma unroll 1
          for (int r = lane; r < kKeys; r += 32) {
            const int p = p0 + r;
            if (p >= far.s.lo && p < far.s.end)
              asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(tc::smem_u32(to + r)),
                           "l"(c.table + (int64_t)far.s.b * c.table_stride + g.page.of(p))
                           : "memory");
            else
              to[r] = -1;
          }
          more = on(far, tf, kPlace);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (at < 0) continue;
        const uint32_t x = (uint32_t)at;
        asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory");
        if (x >= 4) wait(ctl, &ctl.taken[x & 3], ((x >> 2) - 1) & 1);
        __syncwarp();
        const Seg& s = nx.s;
        const int p0 = s.base + (nx.ct + nt) * kKeys;
        int* pages = ctl.page[x & 7];
        Info& f = ctl.tile[x % kInfos];
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
          const int r = lane + 32 * j, p = p0 + r, sl = p - g.page.of(p) * c.page_size, page = pages[r];
          const bool ok = page >= 0 && page < c.n_pages;
          ctl.off[x & 3][r] = ok ? kv_page_offset(c, page) + (int64_t)sl * c.slot_stride + s.hk * c.head_stride : -1;
          if (E8 && !ok) pages[r] = -1;
          const uint32_t word = __ballot_sync(0xffffffffu, ok);
          if (lane == 0) f.valid[j] = word;
        }
        if (lane >= kMine && lane < 4) f.valid[lane] = 0xffffffffu;
        if (lane == 0) {
          f.p0 = p0, f.n = s.n, f.lo = s.lo;
          const bool differ = a.mask && (p0 + kKeys > s.n || (a.window > 0 && p0 < s.lo + 64));
          f.flags = differ ? 1 | (nx.index & 15) << 1 : 0;
          if (nt == 0) ctl.bad[nx.index & 15][0] = ctl.bad[nx.index & 15][1] = 0;
        }
        __syncwarp();
        if (lane == 0) {
          if (E8) tc::mbar_arrive(&ctl.paged[x & 7]);
          tc::mbar_arrive(&ctl.info[x % kInfos]);
          tc::mbar_arrive(&ctl.placed[x & 3]);
        }
        here = on(nx, nt, kPlace);
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
    }
    if constexpr (!E8) if (warp == 11) {
      // ================================================ queries
      const int ch = lane % kChunks;
      Walk<kKeys, kTurn> w(g, ctl.where, share);
      do {
        const Seg& s = w.s;
        const int r0 = s.blk * S::kRows, rows = min(R - r0, S::kRows), qb = w.index % S::kQs;
        if (w.index >= S::kQs) wait(ctl, &ctl.q_empty[qb], (w.index / S::kQs - 1) & 1);
        const T* q = (const T*)a.q + s.b * a.q_seq + (int64_t)s.hk * G * a.q_head + ch * 8;
#pragma unroll 4
        for (int r = lane / kChunks; r < rows; r += 32 / kChunks) {
          const int node = g.group.of(r0 + r);
          copy16(qs + qb * S::kQBytes + (r >> 7) * (128 * 128 * (D / 64)) + chunk_at(r & 127, ch, 128),
                 q + node * a.q_node + (r0 + r - node * G) * a.q_head, true);
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(tc::smem_u32(&ctl.q_full[qb])) : "memory");
      } while (w.next());
      asm volatile("cp.async.wait_all;" ::: "memory");
    }
    if constexpr (E8) if (warp >= 10) {
      // ================================================ scales: of keys, of values
      // What brings a row's scale to the tile's largest, or its own number for the softmax; bytes are loaded a
      // tile ahead.  The codes go to a stage: copies wait their turn here, apart from the warps that widen them.
      constexpr int kMine = kKeys / 32;
      const int which = warp - 10;
      const uint8_t* base = which ? a.sc.v : a.sc.k;
      Walk<kKeys, kTurn> far(g, ctl.where, share);
      int tf = far.ct, b[kMine], next[kMine];
      bool more = true;
      auto load = [&](int (&to)[kMine], uint32_t x) {
        if (!more) return;
        wait(ctl, &ctl.paged[x & 7], (x >> 3) & 1);
        __syncwarp();
        const int* pages = ctl.page[x & 7];
        const uint8_t* head = base + far.s.hk * a.sc.head_stride;
        const int p0 = far.s.base + tf * kKeys;
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
          const int r = lane + 32 * j, p = p0 + r, page = pages[r];
          to[j] = page < 0 || page >= c.n_pages ? -1 : head[page * a.sc.page_stride + (int64_t)(p - g.page.of(p) * c.page_size) * a.sc.slot_stride];
        }
        if (++tf == far.ct + far.cnt) {
          more = far.next();
          tf = far.ct;
        }
      };
      load(b, 0);
#pragma unroll 1
      for (uint32_t x = 0;; ++x) {
        // bytes in [63, 247]; 255 takes no part in the largest and the least
        auto fit = [](int b) { return min(max(b, 63), 247); };
        int big = -1, small = 256;
#pragma unroll
        for (int j = 0; j < kMine; ++j)
          if (b[j] >= 0 && b[j] != 255) big = max(big, fit(b[j])), small = min(small, fit(b[j]));
        big = __reduce_max_sync(0xffffffffu, big);
        small = __reduce_min_sync(0xffffffffu, small);
        Info& f = ctl.tile[x % kInfos];
        const bool columns = (f.flags & 1) || big - small > (which ? 5 : 14);
        if (big < 0) big = 127;
        if (x >= 4) wait(ctl, &ctl.taken[x & 3], ((x >> 2) - 1) & 1);
        if (x >= 8) wait(ctl, &ctl.used[x & 7], ((x >> 3) - 1) & 1);  // so that a wait for a later tile's cannot take one phase for another
        __syncwarp();
#pragma unroll
        for (int j = 0; j < kMine; ++j)
          ctl.fac[x & 3][which][lane + 32 * j] = b[j] < 0 ? 0 : columns ? 0x3c : b[j] == 255 ? 0x7e : (15 + fit(b[j]) - big) << 2;
        if (lane == 0) {
          if (which)
            f.ev = columns ? 0.0f : (float)(big - 127), f.value_columns = columns;
          else
            f.ek = columns ? kRowFactor : __int_as_float(big << 23), f.key_columns = columns;
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&ctl.placed[x & 3]);
        const bool last = !more;
        load(next, x + 1);
        const uint32_t e = 2 * x + which, st = e % S::kStages;
        if (e >= S::kStages) wait(ctl, &ctl.unstaged[st], (e / S::kStages - 1) & 1);
        __syncwarp();
        constexpr int kCh = D / 16, kPass = 32 / kCh, kAtOnce = 4;
        const int64_t* offs = ctl.off[x & 3] + lane / kCh;
        const uint8_t* codes = (const uint8_t*)(which ? c.v : c.k) + lane % kCh * 16;
        const uint32_t dst = ring + kEntries * S::kEntry + st * (S::kEntry / 2) + lane * 16;
#pragma unroll 1
        for (int i0 = 0; i0 < kKeys / kPass; i0 += kAtOnce) {
          int64_t o[kAtOnce];  // read ahead of the copies, which the compiler keeps in their order
#pragma unroll
          for (int y = 0; y < kAtOnce; ++y) o[y] = offs[(i0 + y) * kPass];
#pragma unroll
          for (int y = 0; y < kAtOnce; ++y) copy16(dst + (i0 + y) * 512, codes + (o[y] < 0 ? 0 : o[y]), o[y] >= 0);
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(tc::smem_u32(&ctl.staged[st])) : "memory");
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&ctl.taken[x & 3]);
        if (__builtin_expect(columns, 0)) {
          constexpr uint32_t kSlots = E8 ? S::kScales : 1;
          if (kSlots < 8 && x >= kSlots) wait(ctl, &ctl.used[(x - kSlots) & 7], ((x - kSlots) >> 3) & 1);
          __syncwarp();
          column_scales(reinterpret_cast<float*>(ctl.scale[x % kSlots][which]) + lane, which, kKeys, b[0], b[1], b[2 % kMine], b[3 % kMine]);
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&ctl.info[x % kInfos]);
#pragma unroll
        for (int j = 0; j < kMine; ++j) b[j] = next[j];
        if (last) break;
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
    }
    if (warp == 8) {
    // ================================================== products
      // queries with their sign where the scale is negative
      const uint32_t kIdS = idesc<M>(128, kKeys, 0) | (!E8 && a.scale < 0.0f ? 1u << 13 : 0u), kIdO = idesc<M>(128, D, 1);
      const uint32_t leader = elect(), tm = uniform(tmem);
      const uint64_t k0 = tc::desc_kmajor(0, 1024, tc::kLayoutSW128), v0 = tc::desc_strided(0, kKeys * 128, 1024, tc::kLayoutSW128);
      const uint32_t qs4 = uniform(qs) >> 4, ring4 = uniform(ring) >> 4;  // (addresses of 14 bits: offsets do not carry)
      auto entry = [&](uint32_t e) { return ring4 + (e % kEntries) * (S::kEntry / 16); };
      auto landed = [&](uint32_t e) {
        if (!__all_sync(0xffffffffu, mbar_test(&ctl.full[e % kEntries], (e / kEntries) & 1))) return false;
        // copies write as ordinary stores do, products read through the asynchronous proxy
        if (!E8) tc::fence_async_smem();
        return true;
      };
      auto commit = [&](uint64_t* b) {
        if (leader) tc::mma_commit(b);
      };
      // output of tile t of track x: the weights are there, and the values
      auto outputs = [&](int x, int buf, uint32_t e, bool first) {
        tc::fence_after();
        const uint32_t vd = uniform((uint32_t)v0 | entry(e)), out = tm + S::kO + x * S::kOStep, p = uniform(tm + S::kS + buf * S::kSStep);
        const uint32_t more = uniform(!first);
        constexpr int kIn = S::kGroup / 16;
#pragma unroll
        for (int kk = 0; kk < kKeys / 16; ++kk)
#pragma unroll
          for (int low = 0; low <= kLow; ++low)
            mma_ts(out, p + kk / kIn * S::kGroup + kk % kIn * 8 + low * (S::kGroup / 2), desc_of(vd + kk * 128, (uint32_t)(v0 >> 32)), kIdO,
                   kk + low > 0 ? 1u : more, leader);
        commit(&ctl.pv_done[x]);
      };
      auto scores = [&](int x, int buf, int qb, uint32_t e) {
        tc::fence_after();
        const uint32_t qd = (uint32_t)k0 | (qs4 + (qb * S::kQBytes + x * 128 * 128 * (D / 64)) / 16), kd = uniform((uint32_t)k0 | entry(e));
        const uint32_t to = uniform(tm + S::kS + buf * S::kSStep);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          mma_ss(to, desc_of(qd + ((kk >> 2) * 128 * 128 + (kk & 3) * 32) / 16, (uint32_t)(k0 >> 32)),
                 desc_of(kd + ((kk >> 2) * kKeys * 128 + (kk & 3) * 32) / 16, (uint32_t)(k0 >> 32)), kIdS, kk > 0, leader);
        commit(&ctl.s_full[buf]);
      };
      uint32_t ps[2] = {0, 0};  // phases of the weights
      uint32_t e0 = 0;          // entry of the segment's first keys
      Walk<kKeys, kTurn> w(g, ctl.where, share);
      do {
        const int rows = min(R - w.s.blk * S::kRows, S::kRows), nt = (int)uniform(w.cnt);
        const int qb = S::kQs == 1 ? 0 : (int)uniform(w.index & 1);
        wait(ctl, &ctl.q_full[qb], (w.index / S::kQs) & 1);
        __syncwarp();
        if (!E8) tc::fence_async_smem();
        if constexpr (WIDE) {
          // The tracks take turns: a track's next scores go right behind its outputs, for its softmax is what
          // waits for them.  (Waits in this order wake faster than a look at everything in turn: 400-800 clk.)
          const int tracks = uniform(rows > 128) ? 2 : 1;
          auto await = [&](uint32_t e) {
            wait(ctl, &ctl.full[e % kEntries], (e / kEntries) & 1);
            __syncwarp();
            if (!E8) tc::fence_async_smem();
          };
          await(e0);
          for (int x = 0; x < tracks; ++x) scores(x, x, qb, e0);
          commit(&ctl.empty[e0 % kEntries]);
          if (nt == 1) commit(&ctl.q_empty[qb]);
#pragma unroll 1
          for (int t = 0; t < nt; ++t) {
            const uint32_t ve = e0 + 2 * t + 1, ke = ve + 1;
            await(ve);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              if (x >= tracks) break;
              wait(ctl, &ctl.p_full[x], ps[x] & 1);
              __syncwarp();
              ++ps[x];
              outputs(x, x, ve, t == 0);
              if (x == tracks - 1) commit(&ctl.empty[ve % kEntries]);
              if (t + 1 == nt) continue;
              if (x == 0) await(ke);
              scores(x, x, qb, ke);
              if (x == tracks - 1) {
                commit(&ctl.empty[ke % kEntries]);
                if (t + 2 == nt) commit(&ctl.q_empty[qb]);
              }
            }
          }
        } else {
          int nk = 0, np = 0;  // tiles whose scores, outputs are under way: by what has arrived, scores two tiles ahead
          long long t0 = clock64();
          while (np < nt) {
            bool any = false;
            if (np < nk && __all_sync(0xffffffffu, mbar_test(&ctl.p_full[np & 1], ((np & 1) ? ps[1] : ps[0]) & 1)) &&
                landed(e0 + 2 * np + 1)) {
              if (np & 1)
                ++ps[1];
              else
                ++ps[0];
              const uint32_t e = e0 + 2 * np + 1;
              outputs(0, np & 1, e, np == 0);
              commit(&ctl.empty[e % kEntries]);
              ++np;
              any = true;
            }
            if (nk < nt && nk < np + 2 && landed(e0 + 2 * nk)) {
              const uint32_t e = e0 + 2 * nk;
              scores(0, nk & 1, qb, e);
              commit(&ctl.empty[e % kEntries]);
              if (++nk == nt) commit(&ctl.q_empty[qb]);
              any = true;
            }
            if (any) {
              t0 = clock64();
            } else if (__any_sync(0xffffffffu, clock64() - t0 > ctl.patience || *(volatile int*)&ctl.err)) {
              atomicExch(&ctl.err, 1);
              break;
            }
          }
        }
        e0 += 2 * nt;
      } while (w.next());
      commit(&ctl.fin);
      if (!tc::mbar_wait(&ctl.fin, 0)) atomicExch(&ctl.err, 1);
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
    // ================================================== producers
    // (split, what an entry costs besides its copies is paid side by side)
    constexpr int kN = 32 * S::kBring;
    const int kind = S::kSplit ? (warp - 12) / S::kBring : 0, pt = tid - 384 - kind * kN;
    auto arrive = [&](uint64_t* b) {
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(b);
    };
    // queries of a segment's block of rows (8 bits), by those who bring keys
    auto load_q = [&](const Walk<kKeys, kTurn>& w) {
      if (kind != 0) return;
      const Seg& s = w.s;
      const int hk = s.hk, r0 = s.blk * S::kRows, rows = min(R - r0, S::kRows);
      const int qb = w.index % S::kQs;
      if (w.index >= S::kQs) wait(ctl, &ctl.q_empty[qb], (w.index / S::kQs - 1) & 1);
      __syncwarp();
      const T* q = (const T*)a.q + s.b * a.q_seq + (int64_t)hk * G * a.q_head;
      constexpr int kStep = kN / kChunks;
      const int ch = pt % kChunks;
      auto row_of = [&](int r) {
        const int node = g.group.of(r0 + r);
        return q + node * a.q_node + (r0 + r - node * G) * a.q_head + ch * 8;
      };
      auto place = [&](int r) { return qb * S::kQBytes + (r >> 7) * (128 * 128 * (D / 64)) + chunk_at(r & 127, ch, 128); };
      {
        constexpr int kAtOnce = 4;
#pragma unroll 1
        for (int r1 = 0; r1 < rows; r1 += kAtOnce * kStep) {
          uint4 x[kAtOnce];
#pragma unroll
          for (int u = 0; u < kAtOnce; ++u) {
            const int r = r1 + pt / kChunks + u * kStep;
            x[u] = make_uint4(0, 0, 0, 0);
            if (r < rows) x[u] = *reinterpret_cast<const uint4*>(row_of(r));
          }
#pragma unroll
          for (int u = 0; u < kAtOnce; ++u) {
            const int r = r1 + pt / kChunks + u * kStep;
            uint32_t* y = reinterpret_cast<uint32_t*>(&x[u]);
            // fp16 with the row's largest in [2^14, 2^15), and the scale's sign
            uint32_t most = 0;
            float2 f[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              f[i] = unpack2<T>(y[i]);
              most = max(most, max(__float_as_uint(f[i].x) & 0x7fffffffu, __float_as_uint(f[i].y) & 0x7fffffffu));
            }
#pragma unroll
            for (int i = 1; i < kChunks; i *= 2) most = max(most, __shfl_xor_sync(0xffffffffu, most, i));
            const int ex = (int)(most >> 23);
            const int up = ex == 255 || most == 0 ? 127 : min(268 - ex, 253);  // exponent field of the factor
            const float fac = copysignf(__uint_as_float((uint32_t)up << 23), a.scale);
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = pack2<__half>(f[i].x * fac, f[i].y * fac);
            if (r < rows) {
              if (ch == 0) ctl.qf[w.index % 3][r] = __uint_as_float((uint32_t)(254 - up) << 23);
              *reinterpret_cast<uint4*>(smem + place(r)) = x[u];
            }
          }
        }
        tc::fence_async_smem();
        arrive(&ctl.q_full[qb]);
      }
    };
    Walk<kKeys, kTurn> w(g, ctl.where, share);
    uint32_t tile = 0;  // tiles behind
    auto placed = [&](uint32_t x) {
      wait(ctl, &ctl.placed[x & 3], (x >> 2) & 1);
      __syncwarp();
    };

    if constexpr (!E8) {
      constexpr int kPass = kN / kChunks;  // rows of a pass
      const int row0 = pt / kChunks, ch = pt % kChunks;
      do {
        for (int t = 0; t < w.cnt; ++t, ++tile) {
          placed(tile);
          const int64_t* offs = ctl.off[tile & 3];
          const Info& f = ctl.tile[tile % kInfos];
          static_assert(S::kSplit, "16-bit entries have an even number of places");
          const int kv = kind;
          const uint32_t e = 2 * tile + kv;
          if (e >= kEntries) wait(ctl, &ctl.empty[e % kEntries], (e / kEntries - 1) & 1);
          const uint32_t dst = ring + (e % kEntries) * S::kEntry;
          const T* src = (const T*)(kv ? c.v : c.k) + ch * 8;
          constexpr int kAtOnce = 8;
#pragma unroll 1
          for (int i0 = 0; i0 < kKeys / kPass; i0 += kAtOnce) {
            int64_t o[kAtOnce];  // read ahead of the copies, which the compiler keeps in their order
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) o[i] = offs[row0 + (i0 + i) * kPass];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
              copy16(dst + chunk_at(row0 + (i0 + i) * kPass, ch, kKeys), src + (o[i] < 0 ? 0 : o[i]), o[i] >= 0);
          }
          if (__builtin_expect(kv && (f.flags & 1), 0)) {
            asm volatile("cp.async.wait_all;" ::: "memory");
            clean_values<T, kKeys, kPass>(smem + S::kQs * S::kQBytes + (e % kEntries) * S::kEntry, f, ctl.bad[f.flags >> 1], a.window, a.n_nodes, row0, ch);
            tc::fence_async_smem();
            tc::mbar_arrive(&ctl.full[e % kEntries]);
          } else {
            // the thread arrives when its copies have landed
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(tc::smem_u32(&ctl.full[e % kEntries])) : "memory");
          }
          arrive(&ctl.taken[tile & 3]);
        }
      } while (w.next());
      asm volatile("cp.async.wait_all;" ::: "memory");
    } else {
      // Codes are widened from their stage into the ring
      constexpr int kCh = D / 16, kPass = kN / kCh, kEach = kKeys / kPass;  // 16-code chunks of a row; rows of a pass; of a thread
      constexpr int kStages = S::kStages;
      const int row0 = pt / kCh, ch = pt % kCh;
      unsigned char* stages = smem + S::kQs * S::kQBytes + kEntries * S::kEntry + pt * 16;
      auto put = [&](uint32_t e, const uint8_t* fac, bool check, const Info& f) {
        wait(ctl, &ctl.staged[e % kStages], (e / kStages) & 1);
        if (e >= kEntries) wait(ctl, &ctl.empty[e % kEntries], (e / kEntries - 1) & 1);
        __syncwarp();
        unsigned char* from = stages + (e % kStages) * (S::kEntry / 2);
        if (__builtin_expect(check, 0)) {
          clean_codes<kEach, kPass, kN>(from, f, ctl.bad[f.flags >> 1], a.window, a.n_nodes, row0);
          __syncwarp();  // (a row's lanes are in one warp)
        }
        unsigned char* dst = smem + S::kQs * S::kQBytes + (e % kEntries) * S::kEntry;
        // 8 codes from each half of the row: their chunks of the ring meet no bank twice
        constexpr int kAtOnce = kEach < 4 ? kEach : 4;
        const unsigned char* own = from - pt * 16 + row0 * D + ch * 8;
#pragma unroll 1
        for (int i0 = 0; i0 < kEach; i0 += kAtOnce) {
          uint32_t fr[kAtOnce];
          uint2 z[kAtOnce][2];
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i) {
            fr[i] = fac[row0 + (i0 + i) * kPass] * 0x01000100u;
            z[i][0] = *reinterpret_cast<const uint2*>(own + (i0 + i) * kPass * D);
            z[i][1] = *reinterpret_cast<const uint2*>(own + (i0 + i) * kPass * D + D / 2);
          }
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i) {
            const __half2 ff = *reinterpret_cast<const __half2*>(&fr[i]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint32_t y[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint32_t w = j < 2 ? z[i][h].x : z[i][h].y;
                uint32_t v;
                asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(v) : "h"((uint16_t)(w >> (16 * (j & 1)))));
                const __half2 p = __hmul2(*reinterpret_cast<const __half2*>(&v), ff);
                y[j] = *reinterpret_cast<const uint32_t*>(&p);
              }
              *reinterpret_cast<uint4*>(dst + chunk_at(row0 + (i0 + i) * kPass, ch + h * kCh, kKeys)) = make_uint4(y[0], y[1], y[2], y[3]);
            }
          }
        }
        tc::fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          tc::mbar_arrive(&ctl.full[e % kEntries]);
          tc::mbar_arrive(&ctl.unstaged[e % kStages]);
        }
      };
      do {
        for (int t = 0; t < w.cnt; ++t, ++tile) {
          if (S::kQs == 2 && t == 0) load_q(w);
          placed(tile);
          const Info& f = ctl.tile[tile % kInfos];
#pragma unroll 1
          for (int kv = kind; kv < (S::kSplit ? kind + 1 : 2); ++kv) put(2 * tile + kv, ctl.fac[tile & 3][kv], kv && (f.flags & 1), f);
          arrive(&ctl.taken[tile & 3]);
          // (where they have one place, the first tile is under way before the last segment's are done with)
          if (S::kQs == 1 && t == 0) load_q(w);
        }
      } while (w.next());
    }
  }
  __syncwarp();
  tc::fence_before();
  __syncthreads();
  tc::fence_after();
  if (warp == 8) tc::tmem_dealloc(tmem, 512);
  if (tid == 0 && ctl.err) atomicExch(g.error, 1);
}

// Joins the pieces of a segment in the order of the CTAs.  A warp takes a row; its
// lanes hold the pieces' maxima and sums, then the output's elements.  Bound by
// latency, so the first pieces are on their way before their weights are known.
constexpr int kJoinRows = 8;
template <typename T, typename M, bool E8, int D>
__global__ void __launch_bounds__(32 * kJoinRows) join_kernel(Args g, int block_rows) {
  cudaGridDependencySynchronize();
  cudaTriggerProgrammaticLaunchCompletion();
  const TreeArgs& a = g.a;
  const SegMeta s = g.meta[blockIdx.x];
  if (s.pieces == 0) return;
  const int lane = threadIdx.x & 31, G = a.n_q_heads / a.c.n_heads, R = a.n_nodes * G;
  const int hk = s.group / g.blocks, r0 = s.group % g.blocks * block_rows, row = blockIdx.y * kJoinRows + threadIdx.x / 32;
  if (row >= min(R - r0, block_rows)) return;
  const int64_t slot = (int64_t)block_rows * (D + 2);
  // piece 0 is in first_slot, the others in the first slots of the CTAs after it
  auto at = [&](int i) { return g.part + (i ? (int64_t)((s.first_slot & ~1) + 2 * i) : (int64_t)s.first_slot) * slot; };
  constexpr int kV = D / 128 > 0 ? D / 128 : 1, kEarly = D == 256 ? 4 : 8;  // float4s of a lane (head_dim 64: of half the lanes)
  const bool mine = D > 64 || lane < 16;
  float4 o[kV], early[kEarly][kV];
#pragma unroll
  for (int i = 0; i < kEarly; ++i)
#pragma unroll
    for (int v = 0; v < kV; ++v)
      if (i < s.pieces && mine) early[i][v] = reinterpret_cast<const float4*>(at(i) + (int64_t)row * D)[lane + 32 * v];
  float mm = -CUDART_INF_F, sum = 0.0f, m0 = -CUDART_INF_F, l0 = 0.0f;
  if (lane < s.pieces) {
    m0 = at(lane)[block_rows * D + row];
    l0 = at(lane)[block_rows * (D + 1) + row];
  }
  mm = m0;
  for (int i = lane + 32; i < s.pieces; i += 32) mm = fmaxf(mm, at(i)[block_rows * D + row]);
  for (int x = 16; x; x >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, x));
#pragma unroll
  for (int v = 0; v < kV; ++v) o[v] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  auto add = [&](float4& y, float w, float4 x) {
    y.x = fmaf(w, x.x, y.x), y.y = fmaf(w, x.y, y.y), y.z = fmaf(w, x.z, y.z), y.w = fmaf(w, x.w, y.w);
  };
  for (int i0 = 0; i0 < s.pieces; i0 += 32) {
    if (i0 > 0) {
      m0 = -CUDART_INF_F, l0 = 0.0f;
      if (i0 + lane < s.pieces) {
        m0 = at(i0 + lane)[block_rows * D + row];
        l0 = at(i0 + lane)[block_rows * (D + 1) + row];
      }
    }
    const float f = i0 + lane < s.pieces ? piece_weight(m0, mm) : 0.0f;
    float all = f * l0;
    for (int x = 16; x; x >>= 1) all += __shfl_xor_sync(0xffffffffu, all, x);
    sum += all;
    if (i0 == 0)
#pragma unroll
      for (int i = 0; i < kEarly; ++i) {
        const float w = __shfl_sync(0xffffffffu, f, i);
        if (i < s.pieces && mine)
#pragma unroll
          for (int v = 0; v < kV; ++v) add(o[v], w, early[i][v]);
      }
    const int n = min(32, s.pieces - i0);
#pragma unroll 4
    for (int i = i0 == 0 ? kEarly : 0; i < n; ++i) {
      const float w = __shfl_sync(0xffffffffu, f, i);
      const float4* p = reinterpret_cast<const float4*>(at(i0 + i) + (int64_t)row * D);
#pragma unroll
      for (int v = 0; v < kV; ++v)
        if (mine) add(o[v], w, p[lane + 32 * v]);
    }
  }
  const int rr = r0 + row, node = rr / G, head = hk * G + rr % G;
  T* out = (T*)a.out + s.seq * a.o_seq + node * a.o_node + head * a.o_head;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
  for (int v = 0; v < kV; ++v) {
    if (D == 64 && lane >= 16) continue;
    uint2 x = make_uint2(pack2<T>(o[v].x * inv, o[v].y * inv), pack2<T>(o[v].z * inv, o[v].w * inv));
    if (sum == 0.0f) x = make_uint2(0, 0);
    *reinterpret_cast<uint2*>(out + 4 * (lane + 32 * v)) = x;
  }
  if (a.lse && lane == 0) a.lse[((int64_t)s.seq * a.n_nodes + node) * a.n_q_heads + head] = log_sum<M, E8>(mm, sum);
}

constexpr int64_t kMetaBytes = (kCtas * (int64_t)sizeof(SegMeta) + 255) / 256 * 256;

// Blocks of 256 rows where one of 128 does not hold them all: keys and values are
// brought once for both (256 rows over 16 bits: 242 us; 128 rows alone are 184, and two
// such blocks would be two passes over the cache).  With up to 128 rows a wide block's
// second warpgroup would have nothing to do.
static inline bool wide(int D, int rows) { return D < 256 && rows > 128; }

template <typename T, bool E8, int D, bool WIDE>
static pe_status go(const TreeArgs& a, void* ws, int32_t* error, const Patience& patience, cudaStream_t st) {
  using S = Shape<D, E8, WIDE>;
  using M = typename std::conditional<E8, __half, T>::type;
  const int rows = a.n_nodes * (a.n_q_heads / a.c.n_heads);
  Args g{};
  g.a = a;
  g.blocks = ceil_div(rows, S::kRows);
  g.groups = a.c.n_heads * g.blocks;
  g.page = divisor(a.c.page_size);
  g.group = divisor(a.n_q_heads / a.c.n_heads);
  g.meta = reinterpret_cast<SegMeta*>(ws);
  g.part = reinterpret_cast<float*>(reinterpret_cast<char*>(ws) + kMetaBytes);
  g.error = error;
  g.patience = patience.clocks;
  g.hold = patience.hold;
  // a CTA's tiles are counted in 31 bits
  if ((double)a.c.n_seqs * g.groups * ((double)a.c.max_pages * a.c.page_size / S::kKeys + 2) / kCtas >= 2147483000.0)
    return fail(PE_EINVAL, "n_seqs * n_heads * max_pages * page_size too large");
  auto kern = attn_kernel<T, E8, D, WIDE>;
  PE_TRY_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem));
  PE_TRY_CUDA(launch_pdl(kern, dim3(kCtas), dim3(S::kThreads), S::kSmem, st, true, g));
  PE_TRY_CUDA(launch_pdl(join_kernel<T, M, E8, D>, dim3(kCtas, ceil_div(rows < S::kRows ? rows : S::kRows, kJoinRows)), dim3(32 * kJoinRows), 0, st,
                         true, g, (int)S::kRows));
  return PE_OK;
}

template <typename T, bool E8>
static pe_status go_dim(const TreeArgs& a, void* ws, int32_t* error, const Patience& p, cudaStream_t st) {
  const int rows = a.n_nodes * (a.n_q_heads / a.c.n_heads);
  if (a.c.head_dim == 64) return wide(64, rows) ? go<T, E8, 64, true>(a, ws, error, p, st) : go<T, E8, 64, false>(a, ws, error, p, st);
  if (a.c.head_dim == 128) return wide(128, rows) ? go<T, E8, 128, true>(a, ws, error, p, st) : go<T, E8, 128, false>(a, ws, error, p, st);
  return go<T, E8, 256, false>(a, ws, error, p, st);
}

}  // namespace tree
}  // namespace pe
