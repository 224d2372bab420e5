// Attention with a sliding window and first tokens for prompts: many queries, on
// the 5th-generation tensor cores.
//
// A CTA takes items one after the other, as they come (in equal numbers some got a fifth
// more key tiles than the average of a ragged batch): 2 tiles of up to 128 query rows of a KV
// head (consecutive tokens x the group's query heads, so that a tile spans few
// tokens and reads each key tile once for all heads), over the key tiles that the
// two have in reach, all or a range of them. Roles:
//   warps 0-3, 4-7  softmax of Q tile 0 / 1: a row per thread (= TMEM lane). S is read
//                   into registers, P = 2^(S - m) goes back to TMEM as bf16 pairs, by
//                   halves. Any reference m will do that keeps P and its sums in range
//                   (bf16's is fp32's): the maximum of a row's first tile, moved by the
//                   power of two that a tile's sum of P shows once that passes 2^15, O
//                   with it. So no maximum stands between S and P. l, m and O are fp32.
//                   Then the rows' outputs.
//   warp 8          TMA: Q tiles, K tiles (3 slots), V tiles (2 slots)
//   warp 9          every tcgen05.mma: S_x = Q_x K^T, O_x += P_x V (P from TMEM), the
//                   two Q tiles in turn, across items too
//   warp 10         what the items are, one ahead of the others
//   warp 11         zeros in the rows behind the sequences' last queries
// P enters its product as one bf16 part, rounded by at most 2^-8 of itself: an output
// carries that beside its own rounding. A second part would add half of the products, which bound
// prompts. Calls of one Q tile (up to 128 query rows of a KV head: drafts) have two, so
// that a token is attended as exactly among drafts as alone: their key tiles come from HBM once
// each, 2.8K cycles a tile at the copy rate beside 1.5K of one Q tile's products (1K with one
// part). 64 sequences of 35 rows over 4100 keys take 109 us so, 104 with one part; 256 of 40 over
// 517 keys 63 and 57.7.
//
// Key tiles are 128 rows of the cache. They end where the last query's own key (or
// the ring) ends, so that the only rows in front of the first key are older ones, or
// none, which TMA fills with zeros: no row that never held a token is read. First
// tokens that the window has left make tiles of their own, the last of them as wide
// as they need (in 16s): its products take that share of a tile's.
//
// The products bound it on long windows, under the power limit: 28 heads of 65536 tokens,
// 4096 in reach, take 2.29 ms once (1.63 PFLOP/s) and 2.45 to 2.52 one after the other, 2.06 with no
// softmax between the products. With few key tiles to an item its start and end and the MMA
// warp's look-ups weigh more: 16 prompts of up to 4097 tokens, 512 in reach, 186 us where
// the bytes take 90 and the products 70. A warp of its own for either Q tile's products
// took longer (2.97 ms, 219 us: both tiles' products then finish late), and so did S of a
// tile ahead of the product with P (2.71 ms, 212 us).
#include <atomic>
#include <climits>
#include <type_traits>

#include "common.cuh"
#include "internal.h"
#include "tcgen05.cuh"
#include "window.cuh"

namespace uc {

namespace {

constexpr int kThreads = 384;
constexpr int kQRows = 128;   // rows of a Q tile
constexpr int kKeys = 128;    // keys of a tile
constexpr int kKSlots = 3, kVSlots = 2;
// Registers per thread after the warpgroups rebalance (launch: 168 each). A fourth
// warpgroup for the outputs would leave the softmax 192, and took a tenth longer.
constexpr int kRegSoftmax = 216, kRegOther = 56;
static_assert(2 * 128 * kRegSoftmax + 128 * kRegOther <= kThreads * 168, "register split");
// Tensor memory of Q tile x: S from column 128 x on, and P in its place once its rows are in
// registers (S is written again behind the product that reads P: of one thread's products
// none overtakes another); O.
constexpr uint32_t kColO = 256;
// With P in two parts (one Q tile) P has columns of its own, those that the second tile would have,
// two places in turn: S of a tile is written while the product with P of the one before it
// goes on. The first 64 keys' parts, then the others'.
constexpr uint32_t kColLow = 32;  // (the second part, from the first)
__device__ __forceinline__ uint32_t col_p(int half, uint32_t turn) { return (turn == 0 ? 128u : 384u) + 64 * half; }
constexpr float kNone = -INFINITY;

constexpr int kItemSlots = 2;
constexpr int kLooked = 8;

// What the roles need to know of an item: 2 Q tiles from token t0 on, key tiles j0 ..
// j1 - 1 of those in reach. Tiles below `firsts` hold first tokens (row i of tile j is token
// 128 j + i; tile `whole` has `rest` rows, the others 128); row i of another is at
// position start(j) + i.
struct Item {
  int b, kvh, t0, split;
  int n_query, position;   // of the sequence; of token t0
  int j0, j1;              // j0 < 0: no more items
  int first[2], last[2];   // of each Q tile's tiles (last < first: none)
  int in_first;            // a Q tile takes tiles below this,
  int in_a[2], in_b[2];    // and from in_a to in_b
  int n, whole, rest, firsts;
  int n_a;                 // tiles of the ring's end, before it starts over
  int end_a, end_b;        // positions behind the two parts' last rows
  int low_a, low_b;        // positions from which on their rows are what they seem
  int slot_b;              // the cache's row behind the last
  int in_order;            // the tiles hold every position from 0 on
  int plain_lo, plain_hi;  // tiles of 128 that both Q tiles (or alone: the first) take, neither as its first or last
  int alone;               // the second Q tile takes none
  uint16_t head[kLooked], tail[kLooked];  // todo() of the first and (from behind) the last tiles
  __device__ __forceinline__ bool takes(int x, int j) const {
    return j >= first[x] && j <= last[x] && (j < in_first || (j >= in_a[x] && j <= in_b[x]));
  }
  __device__ __forceinline__ bool part_a(int j) const { return j - firsts < n_a; }
  __device__ __forceinline__ int start(int j) const {
    return part_a(j) ? end_a - kKeys * (n_a - (j - firsts)) : end_b - kKeys * (n - j);
  }
  // the cache's row of a tile's first key (below 0: rows in front of the cache, taken as zeros)
  __device__ __forceinline__ int row(const WindowParams& p, int j) const {
    return j < firsts ? kKeys * j : part_a(j) ? p.n_rows - kKeys * (n_a - (j - firsts)) : slot_b - kKeys * (n - j);
  }
  __device__ __forceinline__ int width(int j) const { return j == whole && rest > 0 ? rest : kKeys; }
  // What is to do for a key tile. Bit x: Q tile x takes it, 2 + x: as its first, 4 + x: as
  // its last; from bit 8: its keys / 16
  __device__ __forceinline__ uint32_t todo(int j) const {
    uint32_t f = (uint32_t)width(j) << 4;
#pragma unroll
    for (int x = 0; x < 2; ++x)
      if (takes(x, j)) f |= (1u << x) | ((uint32_t)(j == first[x]) << (2 + x)) | ((uint32_t)(j == last[x]) << (4 + x));
    return f;
  }
};

__device__ __noinline__ uint32_t todo_of(const Item& it, int j) { return it.todo(j); }

struct PromptSmem {
  uint8_t q[2][2][16384];        // [128 rows][2 x 64 channels], K-major, 128B swizzle
  uint8_t k[kKSlots][2][16384];
  uint8_t v[kVSlots][2][16384];  // (the MN-major B operand)
  uint64_t k_full[kKSlots], k_empty[kKSlots], v_full[kVSlots], v_empty[kVSlots];
  uint64_t q_full[2], q_empty[2], s_full[2], p_full[2][2], o_full[2], o_empty[2], drain;
  uint64_t item_full[kItemSlots], item_empty[kItemSlots];
  Item item[kItemSlots];
  DevStatus status;              // of this CTA's waits
  int loads[4];                  // K, V, Q tile 0 and 1 loads begun
  uint32_t again;                // the last row put aside (of_again), 0: none
  uint32_t tmem_base;
  int begin[kWindowSeqs + 1];    // items before a sequence's
};
static_assert(sizeof(PromptSmem) <= 232448, "shared memory");

__device__ __forceinline__ void item_at(const WindowPromptParams& c, const PromptSmem& sm, int index, Item& it) {
  const WindowParams& p = c.p;
  int lo = 0, hi = p.batch;  // the sequence: begin[lo] <= index < begin[lo + 1]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sm.begin[mid] <= index) lo = mid; else hi = mid;
  }
  it.b = lo;
  const WindowSeq s = window_seq(p, lo);
  const int per = p.n_kv_heads * p.splits, i = index - sm.begin[lo];
  const int blocks = (s.nq + 2 * c.tokens - 1) / (2 * c.tokens);
  it.t0 = (blocks - 1 - i / per) * 2 * c.tokens;  // (the longest first)
  it.kvh = i % per / p.splits;
  it.split = i % per % p.splits;
  it.n_query = s.nq;
  it.position = s.first + it.t0;
  const int pa = it.position, pb = s.first + min(it.t0 + 2 * c.tokens, s.nq) - 1;
  const bool ring = s.kept > 0;
  int from = max(max(pa - p.window + 1, 0), s.kept);
  const int end = max(pb + 1, 0), pad = (p.n_sink + 15) & ~15;
  it.in_order = !ring && from <= pad;
  it.whole = it.rest = it.n_a = 0;
  it.end_a = 0;
  it.low_a = it.low_b = s.kept;
  if (it.in_order) {
    from = 0;
  } else if (end > 0) {
    it.whole = pad / kKeys;
    it.rest = pad % kKeys;
  }
  it.firsts = it.whole + (it.rest > 0);
  int count = max(end - from, 0);
  it.end_b = end;
  it.slot_b = end > 0 ? window_row(p, end - 1) + 1 : 0;
  if (ring && count > 0) {
    const int base = window_row(p, from);
    if (base + count > p.n_rows) {
      const int a = p.n_rows - base;
      it.n_a = (a + kKeys - 1) / kKeys;
      it.end_a = it.low_b = from + a;
      count -= a;
    }
  }
  it.n = it.firsts + it.n_a + (count + kKeys - 1) / kKeys;
  it.j0 = (int)((int64_t)it.n * it.split / p.splits);
  it.j1 = (int)((int64_t)it.n * (it.split + 1) / p.splits);
  if (it.in_order)
    it.in_first = p.n_sink == 0 || it.n == 0 ? 0 : end <= p.n_sink ? it.n : it.n - (end - p.n_sink) / kKeys;
  else
    it.in_first = it.firsts;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int ta = it.t0 + x * c.tokens, tb = min(ta + c.tokens, s.nq) - 1;
    int in_a = it.firsts, in_b = it.n - 1, first = INT_MAX, last = -1;
    if (ta <= tb && s.first + tb >= 0) {
      const int oldest = s.first + ta - p.window + 1, newest = s.first + tb;
      while (in_a < it.n && it.start(in_a) + kKeys <= oldest) ++in_a;
      while (in_b >= it.firsts && it.start(in_b) > newest) --in_b;
      // the first and the last that it takes of j0 .. j1 - 1
      if (it.j0 < min(it.j1, it.in_first)) {
        first = it.j0;
        last = min(it.j1, it.in_first) - 1;
      }
      const int a = max(it.j0, in_a), z = min(it.j1 - 1, in_b);
      if (a <= z) {
        first = min(first, a);
        last = max(last, z);
      }
    }
    it.in_a[x] = in_a;
    it.in_b[x] = in_b;
    it.first[x] = last >= 0 ? first : 0;
    it.last[x] = last;
  }
  it.alone = it.last[1] < it.first[1];
  it.plain_lo = max(max(it.first[0] + 1, it.in_a[0]), it.firsts);
  it.plain_hi = min(it.last[0] - 1, it.in_b[0]);
  if (!it.alone) {
    it.plain_lo = max(it.plain_lo, max(it.first[1] + 1, it.in_a[1]));
    it.plain_hi = min(it.plain_hi, min(it.last[1] - 1, it.in_b[1]));
  }
}

// Bits lo .. hi of 32 (none where hi < lo).
__device__ __forceinline__ uint32_t bits(int lo, int hi) {
  lo = max(lo, 0);
  hi = min(hi, 31);
  return lo > hi ? 0u : (0xffffffffu << lo) & (0xffffffffu >> (31 - hi));
}

__device__ __forceinline__ void tma_4d(void* dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(smem_u32(bar))
      : "memory");
}

// A tile of the cache's rows into a slot, both halves of the channels.
__device__ __forceinline__ void load_keys(uint8_t (*slot)[16384], const CUtensorMap* maps, const Item& it, int j,
                                          const WindowPromptParams& c, uint64_t* bar) {
  const int width = it.width(j);
  const int row = it.row(c.p, j);
  mbar_arrive_expect_tx(bar, 2 * width * 128);
  const CUtensorMap* const map = width == kKeys ? &maps[0] : &maps[1];
  tma_4d(slot[0], map, 0, row, it.kvh, it.b, bar);
  tma_4d(slot[1], map, 64, row, it.kvh, it.b, bar);
}

// Where a row's part of an item's split goes.
__device__ __forceinline__ float* part_of(const WindowParams& p, const Item& it, int row) {
  return p.part + (((int64_t)(it.b * p.n_kv_heads + it.kvh) * p.splits + it.split) * p.group * p.n_tok + row) * (kHeadDim + 4);
}

__device__ __forceinline__ void store_row32(__nv_bfloat16* to, const uint32_t (&o)[32], float inv, bool wide) {
  // 32 values of a row: 64 bytes, in pieces of 32 where they are aligned to them
#pragma unroll
  for (int e = 0; e < 32; e += 16) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      w[i] = pack_bf16(__uint_as_float(o[e + 2 * i]) * inv, __uint_as_float(o[e + 2 * i + 1]) * inv);
    if (wide) {
      asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to + e), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                   "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                   : "memory");
    } else {
      *reinterpret_cast<uint4*>(to + e) = make_uint4(w[0], w[1], w[2], w[3]);
      *reinterpret_cast<uint4*>(to + e + 8) = make_uint4(w[4], w[5], w[6], w[7]);
    }
  }
}

// The bounded waits, in as little code as they take (`aborted`: where one ran out; the
// role's end reports it): the roles' loops are what the instruction caches should hold.
// With the general ones in place 30 % of the warps' time went by fetching.
__device__ __forceinline__ bool wait_some(uint64_t* bar, uint32_t parity, uint64_t lim) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_ns();
#pragma unroll 1
  for (uint32_t it = 1; !mbar_try_wait(bar, parity); ++it)
    if ((it & 15u) == 0u && global_ns() - t0 > lim) return false;
  return true;
}
__device__ __forceinline__ bool wait_lane(uint64_t* bar, uint32_t parity, int where, int& aborted, uint64_t lim) {
  if (wait_some(bar, parity, lim)) return true;
  aborted = where;
  return false;
}
// The same for a converged warp, with one outcome: a vote's, which the compiler knows to
// be the same in every lane (what depends on it may stay in uniform registers).
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, int where, int& aborted, uint64_t lim) {
  const bool ok = __all_sync(0xffffffffu, wait_some(bar, parity, lim));
  if (!ok) aborted = where;
  return ok;
}

// Nothing that reads these is moved in front of this.
__device__ __forceinline__ void tie32(uint32_t (&r)[32]) {
  asm volatile(""
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                 "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]),
                 "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]),
                 "+r"(r[30]), "+r"(r[31]));
}

// Once for the warp, what its lanes have read or written before it.
__device__ __forceinline__ void warp_arrive(uint64_t* bar, int lane) {
  __syncwarp();
  if (lane == 0) mbar_arrive(bar);
}

// Is a row whose outputs are not finite (this lane's query at pos; row_ok: there is one) to be
// computed again? Not where values that it sees are not finite either, in every channel in
// which ones that it does not see, from the same tiles, are: those outputs are its own. Looked at: the
// tiles that the warp's rows see in part, the first and the last kWhole of the others. (Where those hold
// nothing of the kind, sums may have left fp32.)
static __device__ __noinline__ bool not_its_own(const WindowParams& p, const Item& it, int x, int pos, bool row_ok) {
  constexpr int kRun = 8;  // rows in flight
  constexpr int kWhole = 32;
  const int lane = threadIdx.x & 31;
  uint32_t seen[4] = {0u, 0u, 0u, 0u}, unseen[4] = {0u, 0u, 0u, 0u};  // channels 4 l + i: bit l
#pragma unroll 1
  for (int j = it.first[x]; j <= it.last[x]; ++j) {
    if (!it.takes(x, j)) continue;
    const int width = it.width(j), row0 = it.row(p, j);
    int w0 = 0, w1, e0 = 0, e1 = -1;  // the rows that are seen, as in the kernel
    if (j < it.firsts) {
      w1 = min(p.n_sink, pos + 1) - kKeys * j - 1;
    } else {
      const int start = it.start(j);
      w0 = max(pos - p.window + 1, it.part_a(j) ? it.low_a : it.low_b) - start;
      w1 = pos - start;
      if (it.in_order) {
        e0 = -start;
        e1 = min(p.n_sink - 1, pos) - start;
      }
    }
    const bool whole = __all_sync(0xffffffffu, !row_ok || (w0 <= 0 && w1 >= width - 1) || (e0 <= 0 && e1 >= width - 1));
    if (whole && j != it.first[x] && j <= it.last[x] - kWhole) continue;
#pragma unroll 1
    for (int i = 0; i < width; i += kRun) {  // (widths are multiples of 16)
      uint2 w[kRun];
#pragma unroll
      for (int u = 0; u < kRun; ++u) {
        const int row = row0 + i + u;
        w[u] = make_uint2(0u, 0u);
        if (row >= 0 && row < p.n_rows) w[u] = *reinterpret_cast<const uint2*>(p.v.at(it.b, it.kvh, row) + 4 * lane);
      }
#pragma unroll
      for (int u = 0; u < kRun; ++u) {
        const float f[4] = {bf16_lo(w[u].x), bf16_hi(w[u].x), bf16_lo(w[u].y), bf16_hi(w[u].y)};
        if (__all_sync(0xffffffffu, finite(f[0]) && finite(f[1]) && finite(f[2]) && finite(f[3]))) continue;
        const int at = i + u;
        const bool sees = (at >= w0 && at <= w1) || (at >= e0 && at <= e1);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint32_t odd = __ballot_sync(0xffffffffu, !finite(f[c]));
          if (sees)
            seen[c] |= odd;
          else
            unseen[c] |= odd;
        }
      }
    }
  }
  uint32_t any = 0u, alone = 0u;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    any |= seen[c];
    alone |= unseen[c] & ~seen[c];
  }
  return row_ok && (any == 0u || alone != 0u);
}

// Rows that are computed again wait for the end of their CTA's items: key by key they may take
// longer than the waits of its roles for one another do at most (16 heads of 5120 queries behind
// 20000 tokens, one of which takes half of the rows out of range: 129 ms, 0.84 without it). They form
// a list: a row's index and whether its lse is new, plus one, 0 behind the last; the row's first four
// bytes hold the one before it.
constexpr uint32_t kNewLse = 1u << 31;
__device__ __forceinline__ uint32_t of_again(const WindowParams& p, int b, int h, int t, bool new_lse) {
  return (uint32_t)(((int64_t)b * p.n_q_heads + h) * p.n_tok + t + 1) | (new_lse ? kNewLse : 0u);  // (at most 2^30 rows)
}
// By the 8 warps of the softmax, which share a row's keys.
static __device__ __noinline__ void rows_again(const WindowParams& p, uint32_t list, float (*parts)[kHeadDim + 4]) {
  constexpr int kWarps = 8;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll 1
  while (list != 0) {
    const int at = (int)((list & ~kNewLse) - 1), bh = at / p.n_tok, t = at - bh * p.n_tok;
    const int b = bh / p.n_q_heads, h = bh - b * p.n_q_heads;
    const uint32_t before = *reinterpret_cast<const volatile uint32_t*>(p.out.at(b, h, t));
    const WindowPart w = window_row_part(p, b, h, t, warp, kWarps);
    *reinterpret_cast<float4*>(&parts[warp][4 * lane]) = w.o;
    if (lane == 0) *reinterpret_cast<float2*>(&parts[warp][kHeadDim]) = make_float2(w.m, w.l);
    asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory");
    if (warp == 0) {
      WindowPart sum{make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY, 0.f};
      for (int i = 0; i < kWarps; ++i) sum.m = fmaxf(sum.m, parts[i][kHeadDim]);
      const float base = sum.m == -INFINITY ? 0.f : sum.m;
      for (int i = 0; i < kWarps; ++i) {
        const float a = ex2_approx(parts[i][kHeadDim] - base);
        const float4 o = *reinterpret_cast<const float4*>(&parts[i][4 * lane]);
        sum.l = fmaf(a, parts[i][kHeadDim + 1], sum.l);
        sum.o = make_float4(fmaf(a, o.x, sum.o.x), fmaf(a, o.y, sum.o.y), fmaf(a, o.z, sum.o.z), fmaf(a, o.w, sum.o.w));
      }
      const WindowRow y = window_row_of(sum);
      *reinterpret_cast<uint2*>(p.out.at(b, h, t) + 4 * lane) = make_uint2(pack_bf16(y.o.x, y.o.y), pack_bf16(y.o.z, y.o.w));
      if ((list & kNewLse) && lane == 0 && p.lse != nullptr) p.lse[at] = y.lse;
    }
    asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory");
    list = before;
  }
}

// kTwo: one Q tile, P in two bf16 parts. The second Q tile's barriers then serve the first: p_full[t]
// is that of every second tile, t its place of P (a tile's P may be complete before the MMA warp
// asks for that of the one before it: two phases of one barrier could not be told apart), and s_full[1]
// says that a tile's product with P is complete.
template <bool kTwo>
__global__ void __launch_bounds__(kThreads, 1) window_prompt_kernel(const __grid_constant__ WindowPromptParams c) {
  extern __shared__ __align__(1024) uint8_t dyn[];
  PromptSmem& sm = *reinterpret_cast<PromptSmem*>(dyn);
  const WindowParams& p = c.p;
  if ((smem_u32(dyn) & 1023u) != 0) {  // (the swizzled tiles need it)
    if (threadIdx.x == 0) set_status(p.status, UC_ERR_CUDA, 77);
    return;
  }
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kKSlots; ++s) {
      mbar_init(&sm.k_full[s], 1);
      mbar_init(&sm.k_empty[s], 1);
    }
    for (int s = 0; s < kVSlots; ++s) {
      mbar_init(&sm.v_full[s], 1);
      mbar_init(&sm.v_empty[s], 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(&sm.q_full[x], 1);
      mbar_init(&sm.q_empty[x], 1);
      mbar_init(&sm.s_full[x], 1);
      mbar_init(&sm.p_full[x][0], 4);
      mbar_init(&sm.p_full[x][1], 4);
      mbar_init(&sm.o_full[x], 1);
      mbar_init(&sm.o_empty[x], 4);
    }
    for (int s = 0; s < kItemSlots; ++s) {
      mbar_init(&sm.item_full[s], 1);
      mbar_init(&sm.item_empty[s], 10);  // TMA, MMA, 8 warps of softmax
    }
    mbar_init(&sm.drain, 1);
    fence_barrier_init();
    sm.status.code = 0;
    sm.again = 0;
    sm.loads[0] = sm.loads[1] = sm.loads[2] = sm.loads[3] = 0;
  }
  if (warp == 9) tmem_alloc(&sm.tmem_base, 512);
  if (warp == 0) {
    // items before each sequence's: a running sum over lanes
    int before = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
      int n = 0;
      if (b0 + lane < p.batch) {
        const WindowSeq s = window_seq(p, b0 + lane);
        if (blockIdx.x == 0) window_check(p, b0 + lane);
        n = (s.nq + 2 * c.tokens - 1) / (2 * c.tokens) * p.n_kv_heads * p.splits;
      }
      int sum = n;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, sum, d);
        if (lane >= d) sum += y;
      }
      if (b0 + lane < p.batch) sm.begin[b0 + lane] = before + sum - n;
      before += __shfl_sync(0xffffffffu, sum, 31);
    }
    if (lane == 0) sm.begin[p.batch] = before;
  }
  // rows of the Q tiles that no query fills: finite, whatever they are
  for (int i = threadIdx.x; i < 2 * 2 * 16384 / 16; i += kThreads) reinterpret_cast<uint4*>(sm.q)[i] = make_uint4(0, 0, 0, 0);
  fence_proxy_async_smem();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  const int items = sm.begin[p.batch];
  const uint64_t lim = c.p.wait_ns;
  int aborted = 0;

  if (warp >= 8) {
    setmaxnreg_dec<kRegOther>();
    if (warp == 8 && lane == 0) {
      // -------------------------------------------------------------- TMA
      int nk = 0, nv = 0, nq[2] = {0, 0}, load = 0;
      for (uint32_t n = 0; !aborted; ++n) {
        if (!wait_lane(&sm.item_full[n % kItemSlots], (n / kItemSlots) & 1, 79, aborted, lim)) break;
        const Item& it = sm.item[n % kItemSlots];
        if (it.j0 < 0) break;
        // (the first K ahead of Q, whose places come free with the last S of the item before)
        const int j0 = it.j0, j1 = it.j1;
        for (int j = j0; j < max(j1, j0 + 1) && !aborted; ++j) {
          const int ks = nk % kKSlots, vs = nv % kVSlots;
          if (j < j1) {
            if (nk >= kKSlots && !wait_lane(&sm.k_empty[ks], (nk / kKSlots - 1) & 1, 81, aborted, lim)) break;
            if (load++ != c.p.withhold) {
              load_keys(sm.k[ks], c.tk, it, j, c, &sm.k_full[ks]);
              sm.loads[0] = nk + 1;
            }
            ++nk;
          }
          if (j == j0) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              if (it.last[x] < it.first[x]) continue;
              if (nq[x] > 0 && !wait_lane(&sm.q_empty[x], (nq[x] - 1) & 1, 80, aborted, lim)) break;
              mbar_arrive_expect_tx(&sm.q_full[x], 2 * 128 * p.group * c.tokens);
              tma_4d(sm.q[x][0], &c.tq, 0, it.kvh * p.group, it.t0 + x * c.tokens, it.b, &sm.q_full[x]);
              tma_4d(sm.q[x][1], &c.tq, 64, it.kvh * p.group, it.t0 + x * c.tokens, it.b, &sm.q_full[x]);
              sm.loads[2 + x] = ++nq[x];
            }
            if (aborted) break;
          }
          if (j < j1) {
            if (nv >= kVSlots && !wait_lane(&sm.v_empty[vs], (nv / kVSlots - 1) & 1, 82, aborted, lim)) break;
            if (load++ != c.p.withhold) {
              load_keys(sm.v[vs], c.tv, it, j, c, &sm.v_full[vs]);
              sm.loads[1] = nv + 1;
            }
            ++nv;
          }
        }
        mbar_arrive(&sm.item_empty[n % kItemSlots]);
      }
    } else if (warp == 9) {
      // -------------------------------------------------------------- MMA
      const uint32_t lead = elect_one();
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      constexpr uint32_t id_s = idesc_bf16(kQRows, kKeys, 0, 0);
      constexpr uint32_t id_o = idesc_bf16(kQRows, kHeadDim, 0, 1);
      const uint32_t dhi = (uint32_t)(smem_desc_sw128(0, 16) >> 32);
      const uint32_t q_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.q[0][0]), 16);
      const uint32_t k_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.k[0][0]), 16);
      const uint32_t v_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.v[0][0]), 16384);
      constexpr uint32_t kSlotStep = 32768 >> 4;  // descriptor units per slot or Q tile
      int ks = 0, vs = 0;
      uint32_t kph = 0, vph = 0;
      // parities of the next waits by Q tile (bit x); whether O_x has been used
      uint32_t q_par = 0, p_par = 0, o_par = 0, o_any = 0;
      // The next item that has key tiles. With a product of the present one `pending` no
      // item without tiles is looked past: what comes behind it takes the present one's
      // place, which comes free with its last product.
      uint32_t n_item = 0;
      enum { kEnd, kNoTiles, kTiles };
      auto next_item = [&](const Item*& it, bool pending) -> int {
        for (;;) {
          if (!wait_warp(&sm.item_full[n_item % kItemSlots], (n_item / kItemSlots) & 1, 89, aborted, lim)) return kEnd;
          it = &sm.item[n_item % kItemSlots];
          if (it->j0 < 0) return kEnd;
          ++n_item;
          if (it->j0 < it->j1) return kTiles;
          warp_arrive(&sm.item_empty[(n_item - 1) % kItemSlots], lane);
          if (pending) return kNoTiles;
        }
      };
      auto todo = [&](const Item& it, int j, int j0, int j1) -> uint32_t {
        const uint32_t a = (uint32_t)(j - j0), z = (uint32_t)(j1 - 1 - j);
        return a < kLooked ? it.head[a] : z < kLooked ? it.tail[z] : todo_of(it, j);
      };
      // S_x of a tile, with K in slot ks
      auto issue_s = [&](auto plain, uint32_t f, int x) -> bool {
        constexpr bool kIsPlain = decltype(plain)::value;
        if ((kTwo && x == 1) || (!kIsPlain && !(f >> x & 1u))) return true;
        if (!kIsPlain && (f >> (2 + x) & 1u)) {
          if (!wait_warp(&sm.q_full[x], q_par >> x & 1u, 83, aborted, lim)) return false;
          q_par ^= 1u << x;
        }
        const uint32_t q = q_lo + x * kSlotStep, k = k_lo + (uint32_t)ks * kSlotStep;
        if (kIsPlain || (f >> 8 == 8u)) {  // (with constant descriptors and offsets eight of them issue in half the time)
          issue_qk<0>(lead, tm + 128 * x, q, k, dhi, id_s);
        } else {
          const uint32_t id = id_s - ((8u - (f >> 8)) << 18);  // (its N: the tile's keys)
#pragma unroll 1
          for (uint32_t e = 0; e < 8; ++e) {
            const uint32_t at = (e >> 2) * 1024u + (e & 3u) * 2u;
            if (e == 0)
              umma_ss_lead<0, 0, 0>(lead, tm + 128 * x, q, k, dhi, id);
            else
              umma_ss_lead<0, 0, 1>(lead, tm + 128 * x, q + at, k + at, dhi, id);
          }
        }
        umma_commit_lead(lead, &sm.s_full[x]);
        if (!kIsPlain && (f >> (4 + x) & 1u)) umma_commit_lead(lead, &sm.q_empty[x]);
        return true;
      };
      // Two parts: the first or second half of P of the next tile, by its place's barrier.
      uint32_t n_p = 0;  // tiles whose products with P have been issued
      auto wait_p = [&](int half) -> bool {
        if (!wait_warp(&sm.p_full[n_p & 1u][half], n_p >> 1 & 1u, 85, aborted, lim)) return false;
        tc_fence_after();
        return true;
      };
      // O_x += P_x V of a tile. Two parts: of its first and its second 64 keys, x the half. S of the next tile
      // comes between them, as between two Q tiles: it has been read where the first half of P is there.
      auto issue_pv = [&](auto plain, uint32_t f, int x) -> bool {
        constexpr bool kIsPlain = decltype(plain)::value;
        const int qt = kTwo ? 0 : x;
        if (!kIsPlain && !(f >> qt & 1u)) return true;
        const uint32_t again = kIsPlain || !(f >> (2 + qt) & 1u);
        const uint32_t d = tm + kColO + 128 * qt, vb = v_lo + (uint32_t)vs * kSlotStep;
        if (!again && (!kTwo || x == 0) && (o_any >> qt & 1u)) {
          if (!wait_warp(&sm.o_empty[qt], o_par >> qt & 1u, 86, aborted, lim)) return false;
          o_par ^= 1u << qt;
        }
        const uint32_t w = kIsPlain ? 8u : f >> 8;
        if constexpr (kTwo) {
          if (!wait_p(x)) return false;
          const uint32_t a = tm + col_p(x, n_p & 1u), v = vb + 512 * x, n = min(max((int)w - 4 * x, 0), 4);
          const uint32_t acc = again | (uint32_t)x;
          if (n == 4) {
            umma_ts_lead<0>(lead, d, a, v, dhi, id_o, acc);
            umma_ts_lead<1>(lead, d, a, v, dhi, id_o, 1u);
            umma_ts_lead<2>(lead, d, a, v, dhi, id_o, 1u);
            umma_ts_lead<3>(lead, d, a, v, dhi, id_o, 1u);
            umma_ts_lead<0>(lead, d, a + kColLow, v, dhi, id_o, 1u);
            umma_ts_lead<1>(lead, d, a + kColLow, v, dhi, id_o, 1u);
            umma_ts_lead<2>(lead, d, a + kColLow, v, dhi, id_o, 1u);
            umma_ts_lead<3>(lead, d, a + kColLow, v, dhi, id_o, 1u);
          } else {
#pragma unroll 1
            for (uint32_t e = 0; e < n; ++e) {
              umma_ts_lead<0>(lead, d, a + 8 * e, v + 128 * e, dhi, id_o, acc | (uint32_t)(e > 0));
              umma_ts_lead<0>(lead, d, a + kColLow + 8 * e, v + 128 * e, dhi, id_o, 1u);
            }
          }
          if (x == 0) return true;
          ++n_p;
          umma_commit_lead(lead, &sm.s_full[1]);
        } else {
          const uint32_t a = tm + 128 * x, par = p_par >> x & 1u;
          p_par ^= 1u << x;
          if (!wait_warp(&sm.p_full[x][0], par, 85, aborted, lim)) return false;
          tc_fence_after();
          if (w == 8u) {
            umma_ts_lead<0>(lead, d, a, vb, dhi, id_o, again);
            umma_ts_lead<1>(lead, d, a, vb, dhi, id_o, 1u);
            umma_ts_lead<2>(lead, d, a, vb, dhi, id_o, 1u);
            umma_ts_lead<3>(lead, d, a, vb, dhi, id_o, 1u);
            if (!wait_warp(&sm.p_full[x][1], par, 85, aborted, lim)) return false;
            tc_fence_after();
            umma_ts_lead<4>(lead, d, a, vb, dhi, id_o, 1u);
            umma_ts_lead<5>(lead, d, a, vb, dhi, id_o, 1u);
            umma_ts_lead<6>(lead, d, a, vb, dhi, id_o, 1u);
            umma_ts_lead<7>(lead, d, a, vb, dhi, id_o, 1u);
          } else {
#pragma unroll 1
            for (uint32_t e = 0; e < max(w, 5u); ++e) {
              if (e == 4) {
                if (!wait_warp(&sm.p_full[x][1], par, 85, aborted, lim)) return false;
                tc_fence_after();
              }
              if (e < w) umma_ts_lead<0>(lead, d, a + 8 * e, vb + 128 * e, dhi, id_o, again | (uint32_t)(e > 0));
            }
          }
        }
        if (!kIsPlain && (f >> (4 + qt) & 1u)) {
          umma_commit_lead(lead, &sm.o_full[qt]);
          o_any |= 1u << qt;
        }
        return true;
      };
      auto take_k = [&]() { return wait_warp(&sm.k_full[ks], kph, 87, aborted, lim); };
      auto give_k = [&]() {
        umma_commit_lead(lead, &sm.k_empty[ks]);
        if (++ks == kKSlots) {
          ks = 0;
          kph ^= 1u;
        }
      };
      auto give_v = [&]() {
        umma_commit_lead(lead, &sm.v_empty[vs]);
        if (++vs == kVSlots) {
          vs = 0;
          vph ^= 1u;
        }
      };
      auto take_v = [&]() { return wait_warp(&sm.v_full[vs], vph, 88, aborted, lim); };
      constexpr std::true_type kPlain{};
      constexpr std::false_type kAny{};
      // O += P V of a tile, S of the one after it (of the next item, where it was the last).
      // Between plain tiles there is nothing to look up, and elsewhere the next is looked up
      // ahead: with a look at the item in front of each product this warp alone took 3.5K cycles
      // a tile, its products 2K.
      const Item* it;
      int j0 = 0, j = 0, j1 = 0, plain_lo = INT_MAX, plain_hi = 0, alone = 0;
      uint32_t f = 0;  // of tile j; 0: there has been none
      while (!aborted) {
        if (!kTwo && j >= plain_lo && alone) {
          while (j < plain_hi) {
            if (!take_v() || !issue_pv(kPlain, 0, 0)) break;
            give_v();
            if (!take_k() || !issue_s(kPlain, 0, 0)) break;
            give_k();
            f = 0x801;
            ++j;
          }
        } else if (j >= plain_lo) {
          while (j < plain_hi) {
            if (!take_v() || !issue_pv(kPlain, 0, 0) || !take_k() || !issue_s(kPlain, 0, 0) || !issue_pv(kPlain, 0, 1)) break;
            give_v();
            if (!issue_s(kPlain, 0, 1)) break;
            give_k();
            f = kTwo ? 0x801 : 0x803;
            ++j;
          }
        }
        const bool same = j + 1 < j1;
        uint32_t nf = same ? todo(*it, j + 1, j0, j1) : 0u;
        if (aborted || (f && (!take_v() || !issue_pv(kAny, f, 0)))) break;
        int got = kEnd;
        if (same) {
          ++j;
        } else {
          const uint32_t slot = (n_item - 1) % kItemSlots;  // (the present item's)
          got = next_item(it, f != 0);
          if (f) warp_arrive(&sm.item_empty[slot], lane);
          if (got == kTiles) {
            j = j0 = it->j0;
            j1 = it->j1;
            plain_lo = it->plain_lo;
            plain_hi = it->plain_hi;
            alone = it->alone;
            nf = todo(*it, j0, j0, j1);
          }
        }
        if (nf && (!take_k() || !issue_s(kAny, nf, 0))) break;
        if (aborted || (f && !issue_pv(kAny, f, 1))) break;
        if (f) give_v();
        if (!nf) {
          f = 0;
          if (got == kNoTiles) continue;
          break;
        }
        if (!issue_s(kAny, nf, 1)) break;
        give_k();
        f = nf;
      }
    } else if (warp == 10) {
      // ------------------------------------------------------------- items
      for (uint32_t n = 0; !aborted; ++n) {
        const uint32_t slot = n % kItemSlots;
        if (n >= kItemSlots && !wait_warp(&sm.item_empty[slot], (n / kItemSlots - 1) & 1, 78, aborted, lim)) break;
        // the first is its own, the others as they come
        uint32_t taken = 0;
        if (n > 0 && lane == 0) taken = c.taken ? atomicAdd(c.taken, 1u) : n - 1;
        taken = __shfl_sync(0xffffffffu, taken, 0);
        const int64_t index = n == 0 ? blockIdx.x : (int64_t)gridDim.x + (c.taken ? (int64_t)taken : (int64_t)items);
        Item it;
        it.j0 = -1;
        if (index < items) item_at(c, sm, (int)index, it);
        if (lane == 0) sm.item[slot] = it;
        __syncwarp();
        if (lane < kLooked)
          sm.item[slot].head[lane] = (uint16_t)it.todo(it.j0 + lane);
        else if (lane < 2 * kLooked)
          sm.item[slot].tail[lane - kLooked] = (uint16_t)it.todo(it.j1 - 1 - (lane - kLooked));
        warp_arrive(&sm.item_full[slot], lane);
        if (index >= items) break;
      }
    } else if (warp == 11 && p.splits == 1) {
      // ----------------------------------------------- rows behind the queries
      constexpr int kPiece = 32;  // tokens of a head at a time
      const int half = lane >> 4;
      for (int b = 0; b < p.batch; ++b) {
        const int nq = window_seq(p, b).nq, pieces = (p.n_tok - nq + kPiece - 1) / kPiece;
        const int64_t n = (int64_t)pieces * p.n_q_heads;
        for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
          const int h = (int)(i / pieces), t0 = nq + (int)(i - (int64_t)h * pieces) * kPiece;
          __nv_bfloat16* const to = p.out.at(b, h, t0) + 8 * (lane & 15);
          const int m = min(kPiece, p.n_tok - t0);
#pragma unroll 4
          for (int t = half; t < m; t += 2) *reinterpret_cast<uint4*>(to + t * p.out.st) = make_uint4(0u, 0u, 0u, 0u);
          if (lane < m && p.lse != nullptr) p.lse[((int64_t)b * p.n_q_heads + h) * p.n_tok + t0 + lane] = kNone;
        }
      }
    }
  } else {
    setmaxnreg_inc<kRegSoftmax>();
    // ------------------------------------------------------------ softmax
    const int x = warp >> 2, r = threadIdx.x & 127;
    const uint32_t lane_off = (uint32_t)(32 * (warp & 3)) << 16;
    const uint32_t s_col = 128 * x, o_col = kColO + 128 * x;
    const int token = r / p.group, head = r - token * p.group;
    const bool is_row = token < c.tokens;
    const uint64_t sl2_2 = f2_pack(p.scale_log2, p.scale_log2);
    uint32_t n_s = 0, n_o = 0;
    for (uint32_t n = 0; !aborted; ++n) {
      if (!wait_warp(&sm.item_full[n % kItemSlots], (n / kItemSlots) & 1, 94, aborted, lim)) break;
      const Item& it = sm.item[n % kItemSlots];
      if (it.j0 < 0) break;
      const int t = it.t0 + x * c.tokens + token;
      const bool row_ok = is_row && t < it.n_query;
      const int pos = row_ok ? it.position + x * c.tokens + token : -1;
      const int pfirst = it.position + x * c.tokens;
      const int plast = it.position + min((x + 1) * c.tokens, it.n_query - it.t0) - 1;
      float m_ref = kNone, l = 0.f;
      int shift = 0;       // the reference is to move by, before the next tile
      bool alone = false;  // the row left what fp32 holds
      const int first = it.first[x], last = it.last[x], in_a = it.in_a[x], in_b = it.in_b[x], in_first = it.in_first;
      const int firsts = it.firsts, narrow = it.rest > 0 ? it.whole : -1, rest = it.rest;
      const int n_a = it.n_a, a0 = it.end_a - kKeys * (n_a + firsts), b0 = it.end_b - kKeys * it.n;
      const int low_a = it.low_a, low_b = it.low_b;
      const bool in_order = it.in_order;
      const bool any = first <= last;
      constexpr float kFar = 1.2676506e30f;  // 2^100
      // S is complete, and with it every product of O before it (two parts: but the last tile's second half)
      auto begin = [&]() -> bool {
        if (!wait_warp(&sm.s_full[x], n_s & 1, 90, aborted, lim)) return false;
        ++n_s;
        tc_fence_after();
        if (__any_sync(0xffffffffu, shift != 0)) {
          if constexpr (kTwo) {
            if (!wait_warp(&sm.s_full[1], n_s & 1, 95, aborted, lim)) return false;  // (of the tile before, n_s - 2)
            tc_fence_after();
          }
          const float alpha = __uint_as_float((uint32_t)(127 - shift) << 23);
#pragma unroll 1
          for (int cb = 0; cb < 8; ++cb) {
            uint32_t o[16];
            tmem_ld16(tmem + lane_off + o_col + cb * 16, o);
            tmem_wait_ld16(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
            tmem_st16(tmem + lane_off + o_col + cb * 16, o);
          }
          l *= alpha;
          m_ref += (float)shift;
          shift = 0;
        }
        return true;
      };
      auto give = [&](int half) {
        tmem_wait_st();
        tc_fence_before();
        warp_arrive(&sm.p_full[kTwo ? (n_s - 1) & 1 : x][half], lane);
      };
      auto count = [&](float sum) {
        l += sum;
        alone |= sum > kFar;
        if (sum > 32768.f) shift = (int)(__float_as_uint(sum) >> 23) - 127;
      };
      // 2^(s - m) of the first 64 columns as bf16 pairs (low: what they leave of it); acc: sums
      auto form = [&](const uint32_t (&sr)[4][32], uint32_t (&pk)[32], uint32_t (&low)[32], uint64_t (&acc)[2]) {
        const float mb = m_ref == kNone ? 0.f : m_ref;
        const uint64_t nm2 = f2_pack(-mb, -mb);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          float e0f, e1f;
          f2_unpack(f2_fma(f2_pack(__uint_as_float(sr[i >> 4][2 * (i & 15)]), __uint_as_float(sr[i >> 4][2 * (i & 15) + 1])),
                           sl2_2, nm2),
                    e0f, e1f);
          const float a = ex2_approx(e0f), bb = ex2_approx(e1f);
          acc[i & 1] = f2_add(acc[i & 1], f2_pack(a, bb));
          pk[i] = pack_bf16(a, bb);
          if constexpr (kTwo) low[i] = pack_bf16(a - bf16_lo(pk[i]), bb - bf16_hi(pk[i]));
        }
      };
      auto total = [&](const uint64_t (&acc)[2]) {
        float x0, x1;
        f2_unpack(f2_add(acc[0], acc[1]), x0, x1);
        return x0 + x1;
      };
      // A tile. `simple`: every row sees it whole, behind its first: nothing but
      // exponentials between S and P. One copy of the code, its halves in a rolled loop over
      // registers: with copies for each kind of tile and half the warps waited for
      // instructions (16 ragged prompts 233 -> 210 us then).
      auto tile = [&](bool simple, bool fresh, int w0, int w1, int e0, int e1) -> bool {
        if (!begin()) return false;
        uint32_t sr[4][32];
#pragma unroll
        for (int cc = 0; cc < 4; ++cc) tmem_ld32(tmem + lane_off + s_col + 32 * cc, sr[cc]);
        tmem_wait_ld();
#pragma unroll
        for (int cc = 0; cc < 4; ++cc) tie32(sr[cc]);
        if (!simple) {
#pragma unroll
          for (int cc = 0; cc < 4; ++cc) {
            uint32_t see = bits(w0 - 32 * cc, w1 - 32 * cc);
            if (in_order) see |= bits(e0 - 32 * cc, e1 - 32 * cc);
            if (__any_sync(0xffffffffu, see != 0xffffffffu)) {
#pragma unroll
              for (int e = 0; e < 32; ++e)
                if (!(see & (1u << e))) sr[cc][e] = __float_as_uint(kNone);
            }
          }
          if (fresh) {
            // a row's first tile: its maximum is the reference
            float top[2] = {kNone, kNone};
#pragma unroll
            for (int e = 0; e < 128; e += 2)
              top[(e >> 1) & 1] = fmax3(top[(e >> 1) & 1], __uint_as_float(sr[e >> 5][e & 31]),
                                        __uint_as_float(sr[e >> 5][(e & 31) + 1]));
            if (m_ref == kNone) m_ref = fmaxf(top[0], top[1]) * p.scale_log2;
          }
        }
        uint64_t acc[2] = {0ull, 0ull};
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          uint32_t pk[32], low[32];
          form(sr, pk, low, acc);
          if constexpr (kTwo) {
            const uint32_t to = tmem + lane_off + col_p(half, (n_s - 1) & 1);
            tmem_st32(to, pk);
            tmem_st32(to + kColLow, low);
          } else {
            tmem_st32(tmem + lane_off + s_col + 32 * half, pk);
          }
          give(half);
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            sr[0][e] = sr[2][e];
            sr[1][e] = sr[3][e];
          }
        }
        count(total(acc));
        return true;
      };
      for (int j = first; j <= last; ++j) {
        if (j >= in_first && (j < in_a || j > in_b)) continue;
        // which of the tile's rows this row sees
        int w0 = 0, w1, e0 = 0, e1 = -1;
        bool whole;
        if (j < firsts) {
          w1 = min(j == narrow ? rest : kKeys, min(p.n_sink, pos + 1) - kKeys * j) - 1;  // first tokens: rows 0 .. w1
          whole = kKeys * (j + 1) <= min(p.n_sink, pfirst + 1);
        } else {
          const bool a = j - firsts < n_a;
          const int start = (a ? a0 : b0) + kKeys * j, low = a ? low_a : low_b;
          w0 = max(pos - p.window + 1, low) - start;
          w1 = pos - start;
          if (in_order) {
            e0 = max(0, -start);
            e1 = min(p.n_sink - 1, pos) - start;
          }
          whole = start >= max(plast - p.window + 1, low) && start + kKeys - 1 <= pfirst;
        }
        const bool fresh = __any_sync(0xffffffffu, m_ref == kNone);
        if (!tile(whole && !fresh, fresh, whole ? 0 : w0, whole ? kKeys - 1 : w1, e0, e1)) break;
      }
      if (any && (aborted || !wait_warp(&sm.o_full[x], n_o & 1, 91, aborted, lim))) break;
      if (any) ++n_o;
      tc_fence_after();
      // ---------------------------------------------------------- outputs
      const int h = it.kvh * p.group + head;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      __nv_bfloat16* const to = p.out.at(it.b, h, t);
      float* const part = part_of(p, it, t * p.group + head);
      uint64_t odd = 0ull;  // sums of 0 times the outputs: NaN where one is not finite
#pragma unroll 1
      for (int cb = 0; cb < 4; ++cb) {
        uint32_t o[32];
        if (any) {
          tmem_ld32(tmem + lane_off + o_col + cb * 32, o);
          tmem_wait_ld32(o);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0u;
        }
        if (cb == 3 && any) {
          tc_fence_before();
          warp_arrive(&sm.o_empty[x], lane);
        }
        if (!row_ok) continue;
        if (p.splits == 1) {
#pragma unroll
          for (int e = 0; e < 32; e += 2)
            odd = f2_fma(f2_pack(__uint_as_float(o[e]), __uint_as_float(o[e + 1])), 0ull, odd);
          store_row32(to + 32 * cb, o, inv, c.wide_out);
        } else {
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            *reinterpret_cast<uint4*>(part + 32 * cb + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
        }
      }
      float f0, f1;
      f2_unpack(odd, f0, f1);
      if (row_ok && p.splits > 1) {  // (of a row to be taken alone: what the join sees that by)
        if (alone) part[0] = INFINITY;
        *reinterpret_cast<float2*>(part + kHeadDim) = alone ? make_float2(3e38f, INFINITY) : make_float2(m_ref, l);
      } else if (row_ok && p.lse != nullptr) {
        p.lse[((int64_t)it.b * p.n_q_heads + h) * p.n_tok + t] = l == 0.f ? kNone : (m_ref + log2f(l)) * kLn2;
      }
      // rows whose outputs are not finite by no fault of l, nor by what they see: put aside
      bool odd_row = row_ok && p.splits == 1 && !alone && f0 + f1 != 0.f && finite(l);
      if (__any_sync(0xffffffffu, odd_row)) odd_row &= not_its_own(p, it, x, pos, row_ok);
      if (odd_row || (row_ok && p.splits == 1 && alone))
        *reinterpret_cast<uint32_t*>(to) = atomicExch(&sm.again, of_again(p, it.b, h, t, alone));
      warp_arrive(&sm.item_empty[n % kItemSlots], lane);
    }
    tmem_wait_st();
    tc_fence_before();
  }
  if (aborted && (lane == 0 || warp == 8)) set_status(&sm.status, UC_ERR_TIMEOUT, aborted);
  __syncthreads();
  if (sm.status.code != 0) {
    // Where a wait ran out, others may have left with copies and products in
    // flight: neither shared nor tensor memory is given back under them.
    if (threadIdx.x == 0) set_status(p.status, sm.status.code, sm.status.detail);
    bool gone = false;
    if (warp == 8) {
      for (int i = max(0, sm.loads[0] - kKSlots); i < sm.loads[0]; ++i)
        if (2 * i != c.p.withhold) dwait_warp(&sm.k_full[i % kKSlots], (i / kKSlots) & 1, p.status, 92, gone);
      for (int i = max(0, sm.loads[1] - kVSlots); i < sm.loads[1]; ++i)
        if (2 * i + 1 != c.p.withhold) dwait_warp(&sm.v_full[i % kVSlots], (i / kVSlots) & 1, p.status, 92, gone);
      for (int x = 0; x < 2; ++x)
        if (sm.loads[2 + x] > 0) dwait_warp(&sm.q_full[x], (sm.loads[2 + x] - 1) & 1, p.status, 92, gone);
    } else if (warp == 9) {
      umma_commit_lead(elect_one(), &sm.drain);
      dwait_warp(&sm.drain, 0, p.status, 93, gone);
    }
    __syncthreads();
  } else if (warp < 8 && sm.again != 0) {
    rows_again(p, sm.again, reinterpret_cast<float(*)[kHeadDim + 4]>(sm.q));
  }
  if (warp == 9) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

}  // namespace

void launch_window_prompt(const WindowPromptParams& c, int grid, cudaStream_t st) {
  static std::atomic<uint64_t> set[2];
  const auto kernel = c.two_parts ? window_prompt_kernel<true> : window_prompt_kernel<false>;
  allow_smem(kernel, sizeof(PromptSmem), &set[c.two_parts]);
  kernel<<<grid, kThreads, sizeof(PromptSmem), st>>>(c);
  count_launch();
  if (c.p.splits > 1) launch_window_join(c.p, st);
}

}  // namespace uc
