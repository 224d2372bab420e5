// Attention with a sliding window and first tokens for prompts: many queries, on
// the 5th-generation tensor cores.
//
// A CTA takes items one after the other: 2 tiles of up to 128 query rows of a KV
// head (consecutive tokens x the group's query heads, so that a tile spans few
// tokens and reads each key tile once for all heads), over the key tiles that the
// two have in reach, all or a range of them. Roles:
//   warps 0-3, 4-7  softmax of Q tile 0 / 1: a row per thread (= TMEM lane). S is read
//                   into registers, P = 2^(S - m) goes back to TMEM as bf16 pairs; the
//                   reference m moves only when a row's maximum passes it by 2^8, and
//                   O is scaled then; l, m and O are fp32. Then the rows' outputs.
//   warp 8          TMA: Q tiles, K tiles (3 slots), V tiles (2 slots)
//   warp 9          every tcgen05.mma: S_x = Q_x K^T, O_x += P_x V (P from TMEM), the
//                   two Q tiles in turn, across items too
//   warps 10, 11    zeros in the rows behind the sequences' last queries
// P enters its product as one bf16 part, rounded by at most 2^-8 of itself: an output
// carries that beside its own rounding.
//
// Key tiles are 128 rows of the cache. They end where the last query's own key (or
// the ring) ends, so that the only rows in front of the first key are older ones, or
// none, which TMA fills with zeros: no row that never held a token is read. First
// tokens that the window has left lie in the first rows of the first tile(s), by a
// copy of their own, in place of such rows.
#include <climits>
#include <mutex>

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
// Registers per thread after the warpgroups rebalance (launch: 168 each).
constexpr int kRegSoftmax = 216, kRegOther = 56;
static_assert(2 * 128 * kRegSoftmax + 128 * kRegOther <= kThreads * 168, "register split");
// Tensor memory: one S for both Q tiles (a row is in registers long before the other
// tile's S is due), P and O of each.
constexpr uint32_t kColP = 128, kColO = 256;
constexpr float kNone = -INFINITY;

struct PromptSmem {
  uint8_t q[2][2][16384];        // [128 rows][2 x 64 channels], K-major, 128B swizzle
  uint8_t k[kKSlots][2][16384];
  uint8_t v[kVSlots][2][16384];  // (the MN-major B operand)
  uint64_t k_full[kKSlots], k_empty[kKSlots], v_full[kVSlots], v_empty[kVSlots];
  uint64_t q_full[2], q_empty[2], s_full[2], s_free[2], p_full[2], o_full[2], o_empty[2], drain;
  DevStatus status;              // of this CTA's waits
  int loads[4];                  // K, V, Q tile 0 and 1 loads begun
  uint32_t tmem_base;
  int begin[kWindowSeqs + 1];    // items before a sequence's
};
static_assert(sizeof(PromptSmem) + 1024 <= 232448, "shared memory");

// The key tiles of an item, and where their rows come from. Tile j has rows of
// first tokens 128 j .. while j < whole (128 of them) and `rest` in tile `whole`;
// its other rows are row i at position start(j) + i.
struct KeyTiles {
  int n;              // tiles
  int whole, rest;    // tiles of first tokens alone; rows of them in the next
  int n_a;            // tiles of the ring's end, before it starts over
  int end_a, end_b;   // positions behind the two parts' last rows
  int low_a, low_b;   // positions from which on their rows are what they seem
  int slot_b;         // the cache's row behind the last
  int sinks;          // keys below this are seen whatever the window
  bool in_order;      // the tiles hold every position from 0 on
  __device__ __forceinline__ int start(int j) const {
    return j - whole < n_a ? end_a - kKeys * (n_a - (j - whole)) : end_b - kKeys * (n - j);
  }
  __device__ __forceinline__ int low(int j) const { return j - whole < n_a ? low_a : low_b; }
};

struct Item {
  int b, kvh, split, t0;
  WindowSeq s;
  int j0, j1;                    // this item's key tiles
  int first[2], last[2];         // of each Q tile's (last < first: none)
  int in_sinks, in_a[2], in_b[2];  // a Q tile takes tiles below in_sinks, and from in_a to in_b
  __device__ __forceinline__ bool takes(int x, int j) const {
    return j >= first[x] && j <= last[x] && (j < in_sinks || (j >= in_a[x] && j <= in_b[x]));
  }
};

__device__ __forceinline__ void item_at(const WindowPromptParams& c, const PromptSmem& sm, int index, Item& it,
                                        KeyTiles& k) {
  const WindowParams& p = c.p;
  int lo = 0, hi = p.batch;  // the sequence: begin[lo] <= index < begin[lo + 1]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sm.begin[mid] <= index) lo = mid; else hi = mid;
  }
  it.b = lo;
  it.s = window_seq(p, lo);
  const int per = p.n_kv_heads * p.splits, i = index - sm.begin[lo];
  const int blocks = (it.s.nq + 2 * c.tokens - 1) / (2 * c.tokens);
  it.t0 = (blocks - 1 - i / per) * 2 * c.tokens;  // (the longest first)
  it.kvh = i % per / p.splits;
  it.split = i % per % p.splits;
  const int pa = it.s.first + it.t0, pb = it.s.first + min(it.t0 + 2 * c.tokens, it.s.nq) - 1;
  const bool ring = it.s.kept > 0;
  int from = max(max(pa - p.window + 1, 0), it.s.kept);
  const int end = max(pb + 1, 0), pad = (p.n_sink + 7) & ~7;
  k.in_order = !ring && from <= pad;
  k.sinks = p.n_sink;
  k.whole = k.rest = k.n_a = 0;
  k.end_a = 0;
  k.low_a = k.low_b = it.s.kept;
  if (k.in_order) {
    from = 0;
  } else {
    k.whole = pad / kKeys;
    k.rest = pad % kKeys;
  }
  int count = max(end - from, 0);
  k.end_b = end;
  if (end == 0) {
    k.n = k.whole = k.rest = 0;
    k.slot_b = 0;
  } else {
    k.slot_b = window_row(p, end - 1) + 1;
    int head = k.rest;  // rows that the first part's tiles hold beside its keys
    if (ring && count > 0) {
      const int base = window_row(p, from);
      if (base + count > p.n_rows) {
        const int a = p.n_rows - base;
        k.n_a = (a + head + kKeys - 1) / kKeys;
        k.end_a = k.low_b = from + a;
        count -= a;
        head = 0;
      }
    }
    k.n = k.whole + k.n_a + (count + head + kKeys - 1) / kKeys;
  }
  it.j0 = (int)((int64_t)k.n * it.split / p.splits);
  it.j1 = (int)((int64_t)k.n * (it.split + 1) / p.splits);
  if (k.in_order)
    it.in_sinks = p.n_sink == 0 || k.n == 0 ? 0 : end <= p.n_sink ? k.n : k.n - (end - p.n_sink) / kKeys;
  else
    it.in_sinks = k.whole + (k.rest > 0);
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int ta = it.t0 + x * c.tokens, tb = min(ta + c.tokens, it.s.nq) - 1;
    it.first[x] = 0;
    it.last[x] = -1;
    it.in_a[x] = k.whole;
    it.in_b[x] = k.n - 1;
    if (ta > tb || it.s.first + tb < 0) continue;
    const int oldest = it.s.first + ta - p.window + 1, newest = it.s.first + tb;
    while (it.in_a[x] < k.n && k.start(it.in_a[x]) + kKeys <= oldest) ++it.in_a[x];
    while (it.in_b[x] >= k.whole && k.start(it.in_b[x]) > newest) --it.in_b[x];
    // the first and the last that it takes of j0 .. j1 - 1
    int first = INT_MAX, last = -1;
    if (it.j0 < min(it.j1, it.in_sinks)) {
      first = it.j0;
      last = min(it.j1, it.in_sinks) - 1;
    }
    const int a = max(it.j0, it.in_a[x]), z = min(it.j1 - 1, it.in_b[x]);
    if (a <= z) {
      first = min(first, a);
      last = max(last, z);
    }
    if (last >= 0) {
      it.first[x] = first;
      it.last[x] = last;
    }
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
__device__ __forceinline__ void load_keys(uint8_t (*slot)[16384], const CUtensorMap* maps, const KeyTiles& k, int j,
                                          const WindowPromptParams& c, const Item& it, uint64_t* bar) {
  mbar_arrive_expect_tx(bar, 2 * kKeys * 128);
  const bool a = j - k.whole < k.n_a;
  const int row = j < k.whole ? kKeys * j : a ? c.p.n_rows - kKeys * (k.n_a - (j - k.whole)) : k.slot_b - kKeys * (k.n - j);
  const int rest = j == k.whole ? k.rest : 0;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (rest == 0) {
      tma_4d(slot[half], &maps[0], 64 * half, row, it.kvh, it.b, bar);
    } else {
      tma_4d(slot[half], &maps[1], 64 * half, kKeys * k.whole, it.kvh, it.b, bar);
      tma_4d(slot[half] + 128 * rest, &maps[2], 64 * half, row + rest, it.kvh, it.b, bar);
    }
  }
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

__global__ void __launch_bounds__(kThreads, 1) window_prompt_kernel(const __grid_constant__ WindowPromptParams c) {
  extern __shared__ uint8_t dyn[];
  PromptSmem& sm = *reinterpret_cast<PromptSmem*>((reinterpret_cast<uintptr_t>(dyn) + 1023) & ~static_cast<uintptr_t>(1023));
  const WindowParams& p = c.p;
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
      mbar_init(&sm.s_free[x], kQRows);
      mbar_init(&sm.p_full[x], kQRows);
      mbar_init(&sm.o_full[x], 1);
      mbar_init(&sm.o_empty[x], kQRows);
    }
    mbar_init(&sm.drain, 1);
    fence_barrier_init();
    sm.status.code = 0;
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
  DevStatus* const st = &sm.status;
  const uint64_t lim = c.wait_ns;
  bool aborted = false;

  if (warp >= 8) {
    setmaxnreg_dec<kRegOther>();
    if (warp == 8 && lane == 0) {
      // -------------------------------------------------------------- TMA
      int nk = 0, nv = 0, nq[2] = {0, 0}, load = 0;
      for (int i = blockIdx.x; i < items && !aborted; i += gridDim.x) {
        Item it;
        KeyTiles k;
        item_at(c, sm, i, it, k);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          if (it.last[x] < it.first[x]) continue;
          if (nq[x] > 0 && !dwait(&sm.q_empty[x], (nq[x] - 1) & 1, st, 80, aborted, lim)) break;
          mbar_arrive_expect_tx(&sm.q_full[x], 2 * 128 * p.group * c.tokens);
          tma_4d(sm.q[x][0], &c.tq, 0, it.kvh * p.group, it.t0 + x * c.tokens, it.b, &sm.q_full[x]);
          tma_4d(sm.q[x][1], &c.tq, 64, it.kvh * p.group, it.t0 + x * c.tokens, it.b, &sm.q_full[x]);
          sm.loads[2 + x] = ++nq[x];
        }
        for (int j = it.j0; j < it.j1 && !aborted; ++j) {
          const int ks = nk % kKSlots, vs = nv % kVSlots;
          if (nk >= kKSlots && !dwait(&sm.k_empty[ks], (nk / kKSlots - 1) & 1, st, 81, aborted, lim)) break;
          if (load++ != c.withhold) {
            load_keys(sm.k[ks], c.tk, k, j, c, it, &sm.k_full[ks]);
            sm.loads[0] = nk + 1;
          }
          ++nk;
          if (nv >= kVSlots && !dwait(&sm.v_empty[vs], (nv / kVSlots - 1) & 1, st, 82, aborted, lim)) break;
          if (load++ != c.withhold) {
            load_keys(sm.v[vs], c.tv, k, j, c, it, &sm.v_full[vs]);
            sm.loads[1] = nv + 1;
          }
          ++nv;
        }
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
      uint32_t q_seen[2] = {0, 0}, s_done[2] = {0, 0}, p_done[2] = {0, 0}, o_done[2] = {0, 0};  // events so far
      int s_last = -1;  // the Q tile whose S came last
      Item cur, nxt;
      // the first tile of the next item that has any, from item i on
      auto find = [&](int i, Item& it) {
        for (; i < items; i += gridDim.x) {
          KeyTiles k;
          item_at(c, sm, i, it, k);
          if (it.j0 < it.j1) break;
        }
        return i;
      };
      // S_x of tile j of an item, with K in slot ks
      auto issue_s = [&](const Item& it, int x, int j) -> bool {
        if (!it.takes(x, j)) return true;
        if (j == it.first[x]) {
          if (!dwait_warp(&sm.q_full[x], q_seen[x] & 1, st, 83, aborted, lim)) return false;
          ++q_seen[x];
        }
        if (s_last >= 0 && !dwait_warp(&sm.s_free[s_last], (s_done[s_last] - 1) & 1, st, 84, aborted, lim)) return false;
        tc_fence_after();
        issue_qk<0>(lead, tm, q_lo + x * kSlotStep, k_lo + (uint32_t)ks * kSlotStep, dhi, id_s);
        umma_commit_lead(lead, &sm.s_full[x]);
        if (j == it.last[x]) umma_commit_lead(lead, &sm.q_empty[x]);
        ++s_done[x];
        s_last = x;
        return true;
      };
      auto issue_pv = [&](const Item& it, int x, int j) -> bool {
        if (!it.takes(x, j)) return true;
        if (!dwait_warp(&sm.p_full[x], p_done[x] & 1, st, 85, aborted, lim)) return false;
        ++p_done[x];
        if (j == it.first[x] && o_done[x] > 0 &&
            !dwait_warp(&sm.o_empty[x], (o_done[x] - 1) & 1, st, 86, aborted, lim))
          return false;
        tc_fence_after();
        const uint32_t d = tm + kColO + 128 * x, a = tm + kColP + 64 * x, vb = v_lo + (uint32_t)vs * kSlotStep;
        umma_ts_lead<0>(lead, d, a, vb, dhi, id_o, j > it.first[x]);
        umma_ts_lead<1>(lead, d, a, vb, dhi, id_o, 1u);
        umma_ts_lead<2>(lead, d, a, vb, dhi, id_o, 1u);
        umma_ts_lead<3>(lead, d, a, vb, dhi, id_o, 1u);
        umma_ts_lead<4>(lead, d, a, vb, dhi, id_o, 1u);
        umma_ts_lead<5>(lead, d, a, vb, dhi, id_o, 1u);
        umma_ts_lead<6>(lead, d, a, vb, dhi, id_o, 1u);
        umma_ts_lead<7>(lead, d, a, vb, dhi, id_o, 1u);
        if (j == it.last[x]) {
          umma_commit_lead(lead, &sm.o_full[x]);
          ++o_done[x];
        }
        return true;
      };
      auto take_k = [&]() { return dwait_warp(&sm.k_full[ks], kph, st, 87, aborted, lim); };
      auto give_k = [&]() {
        umma_commit_lead(lead, &sm.k_empty[ks]);
        if (++ks == kKSlots) {
          ks = 0;
          kph ^= 1u;
        }
      };
      int i = find(blockIdx.x, cur), j = cur.j0;
      if (i < items) {
        if (take_k() && issue_s(cur, 0, j) && issue_s(cur, 1, j)) give_k();
        while (!aborted) {
          // the tile after this one
          bool more = true, same = j + 1 < cur.j1;
          int ni = i;
          if (!same) {
            ni = find(i + gridDim.x, nxt);
            more = ni < items;
          }
          if (!dwait_warp(&sm.v_full[vs], vph, st, 88, aborted, lim)) break;
          if (!issue_pv(cur, 0, j)) break;
          if (more) {
            if (!take_k()) break;
            if (!(same ? issue_s(cur, 0, j + 1) : issue_s(nxt, 0, nxt.j0))) break;
          }
          if (!issue_pv(cur, 1, j)) break;
          umma_commit_lead(lead, &sm.v_empty[vs]);
          if (++vs == kVSlots) {
            vs = 0;
            vph ^= 1u;
          }
          if (!more) break;
          if (!(same ? issue_s(cur, 1, j + 1) : issue_s(nxt, 1, nxt.j0))) break;
          give_k();
          if (same) {
            ++j;
          } else {
            cur = nxt;
            i = ni;
            j = cur.j0;
          }
        }
      }
    } else if (warp >= 10 && p.splits == 1) {
      // ----------------------------------------------- rows behind the queries
      for (int b = 0; b < p.batch; ++b) {
        const int nq = window_seq(p, b).nq;
        const int64_t n = (int64_t)(p.n_tok - nq) * p.n_q_heads;
        for (int64_t r = blockIdx.x * 2 + (warp - 10); r < n; r += 2 * gridDim.x) {
          const int t = nq + (int)(r / p.n_q_heads), h = (int)(r % p.n_q_heads);
          *reinterpret_cast<uint2*>(p.out.at(b, h, t) + 4 * lane) = make_uint2(0u, 0u);
          if (lane == 0 && p.lse != nullptr) p.lse[((int64_t)b * p.n_q_heads + h) * p.n_tok + t] = kNone;
        }
      }
    }
  } else {
    setmaxnreg_inc<kRegSoftmax>();
    // ------------------------------------------------------------ softmax
    const int x = warp >> 2, r = threadIdx.x & 127;
    const uint32_t lane_off = (uint32_t)(32 * (warp & 3)) << 16;
    const uint32_t p_col = kColP + 64 * x, o_col = kColO + 128 * x;
    const int token = r / p.group, head = r - token * p.group;
    const bool is_row = token < c.tokens;
    const uint64_t sl2_2 = f2_pack(p.scale_log2, p.scale_log2);
    uint32_t n_s = 0, n_o = 0;
    for (int i = blockIdx.x; i < items && !aborted; i += gridDim.x) {
      Item it;
      KeyTiles k;
      item_at(c, sm, i, it, k);
      const int t = it.t0 + x * c.tokens + token;
      const bool row_ok = is_row && t < it.s.nq;
      const int pos = row_ok ? it.s.first + t : -1;
      const int pfirst = it.s.first + it.t0 + x * c.tokens;
      const int plast = it.s.first + min(it.t0 + (x + 1) * c.tokens, it.s.nq) - 1;
      float m_ref = kNone, l = 0.f;
      const int first = x ? it.first[1] : it.first[0], last = x ? it.last[1] : it.last[0];
      const int in_a = x ? it.in_a[1] : it.in_a[0], in_b = x ? it.in_b[1] : it.in_b[0];
      const bool any = first <= last;
      for (int j = first; j <= last; ++j) {
        if (j >= it.in_sinks && (j < in_a || j > in_b)) continue;
        if (!dwait_warp(&sm.s_full[x], n_s & 1, st, 90, aborted, lim)) break;
        ++n_s;
        tc_fence_after();
        uint32_t sr[4][32];
#pragma unroll
        for (int cc = 0; cc < 4; ++cc) tmem_ld32(tmem + lane_off + 32 * cc, sr[cc]);
        tmem_wait_ld();
        tc_fence_before();
        mbar_arrive(&sm.s_free[x]);
        // which of the tile's rows this row sees
        const int start = k.start(j), low = k.low(j);
        const int head_rows = j < k.whole ? kKeys : j == k.whole ? k.rest : 0;
        const bool whole = head_rows == 0 ? start >= max(plast - p.window + 1, low) && start + kKeys - 1 <= pfirst
                                          : head_rows == kKeys && kKeys * (j + 1) <= min(p.n_sink, pfirst + 1);
        if (!whole) {
          const int s1 = min(head_rows, min(p.n_sink, pos + 1) - kKeys * min(j, k.whole)) - 1;  // first tokens: rows 0 .. s1
          const int w0 = max(max(pos - p.window + 1, low) - start, head_rows), w1 = head_rows == kKeys ? -1 : pos - start;
          const int e0 = k.in_order ? max(0, -start) : 0, e1 = k.in_order ? min(p.n_sink - 1, pos) - start : -1;
#pragma unroll
          for (int cc = 0; cc < 4; ++cc) {
            const uint32_t see = bits(-32 * cc, s1 - 32 * cc) | bits(w0 - 32 * cc, w1 - 32 * cc) |
                                 bits(e0 - 32 * cc, e1 - 32 * cc);
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (!(see >> e & 1u)) sr[cc][e] = __float_as_uint(kNone);
          }
        }
        float mx[4] = {kNone, kNone, kNone, kNone};
#pragma unroll
        for (int c2 = 0; c2 < kKeys / 2; ++c2)
          mx[c2 & 3] = fmax3(mx[c2 & 3], __uint_as_float(sr[(2 * c2) >> 5][(2 * c2) & 31]),
                             __uint_as_float(sr[(2 * c2 + 1) >> 5][(2 * c2 + 1) & 31]));
        const float tmax = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.scale_log2;
        const bool grow = tmax > m_ref + 8.f;
        if (__any_sync(0xffffffffu, grow)) {
          const float m_new = grow ? tmax : m_ref;
          const bool need_o = grow && m_ref != kNone;
          if (__any_sync(0xffffffffu, need_o)) {
            // O is final: its last product was issued before this S
            const float alpha = need_o ? ex2_approx(m_ref - m_new) : 1.f;
#pragma unroll 1
            for (int cb = 0; cb < 8; ++cb) {
              uint32_t o[16];
              tmem_ld16(tmem + lane_off + o_col + cb * 16, o);
              tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
              tmem_st16(tmem + lane_off + o_col + cb * 16, o);
            }
            l *= alpha;
          }
          m_ref = m_new;
        }
        const float mb = m_ref == kNone ? 0.f : m_ref;
        const uint64_t nm2 = f2_pack(-mb, -mb);
        uint32_t pk[2][32];
        uint64_t acc[2] = {0ull, 0ull};
#pragma unroll
        for (int c2 = 0; c2 < kKeys / 2; ++c2) {
          float e0, e1;
          f2_unpack(f2_fma(f2_pack(__uint_as_float(sr[(2 * c2) >> 5][(2 * c2) & 31]),
                                   __uint_as_float(sr[(2 * c2 + 1) >> 5][(2 * c2 + 1) & 31])),
                           sl2_2, nm2),
                    e0, e1);
          const float a = ex2_approx(e0), bb = ex2_approx(e1);
          acc[c2 & 1] = f2_add(acc[c2 & 1], f2_pack(a, bb));
          pk[c2 >> 5][c2 & 31] = pack_bf16(a, bb);
        }
        tmem_st32(tmem + lane_off + p_col, pk[0]);
        tmem_st32(tmem + lane_off + p_col + 32, pk[1]);
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&sm.p_full[x]);
        float sum[4];
        f2_unpack(acc[0], sum[0], sum[1]);
        f2_unpack(acc[1], sum[2], sum[3]);
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      }
      if (any && (aborted || !dwait_warp(&sm.o_full[x], n_o & 1, st, 91, aborted, lim))) break;
      if (any) ++n_o;
      tc_fence_after();
      // ---------------------------------------------------------- outputs
      const int h = it.kvh * p.group + head;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      __nv_bfloat16* const to = p.out.at(it.b, h, t);
      float* const part = p.part + (((int64_t)(it.b * p.n_kv_heads + it.kvh) * p.splits + it.split) * p.group * p.n_tok +
                                    (int64_t)t * p.group + head) * (kHeadDim + 4);
      uint64_t odd = 0ull;  // sums of 0 times the outputs: NaN where one is not finite
#pragma unroll 1
      for (int cb = 0; cb < 4; ++cb) {
        uint32_t o[32];
        if (any) {
          tmem_ld32(tmem + lane_off + o_col + cb * 32, o);
          tmem_wait_ld();
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0u;
        }
        if (cb == 3 && any) {
          tc_fence_before();
          mbar_arrive(&sm.o_empty[x]);
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
      if (row_ok && p.splits == 1) {
        if (p.lse != nullptr)
          p.lse[((int64_t)it.b * p.n_q_heads + h) * p.n_tok + t] = l == 0.f ? kNone : (m_ref + log2f(l)) * kLn2;
      } else if (row_ok) {
        *reinterpret_cast<float2*>(part + kHeadDim) = make_float2(m_ref, l);
      }
      // rows whose outputs are not finite by no fault of l: from the definition
      uint32_t again = __ballot_sync(0xffffffffu, row_ok && p.splits == 1 && f0 + f1 != 0.f && finite(l));
      for (; again; again &= again - 1) {
        const int from = __ffs(again) - 1;
        const int ah = __shfl_sync(0xffffffffu, h, from), at = __shfl_sync(0xffffffffu, t, from);
        const float4 y = window_row_alone(p, it.b, ah, at);
        *reinterpret_cast<uint2*>(p.out.at(it.b, ah, at) + 4 * lane) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
      }
    }
    tmem_wait_st();
    tc_fence_before();
  }
  __syncthreads();
  if (sm.status.code != 0) {
    // Where a wait ran out, others may have left with copies and products in
    // flight: neither shared nor tensor memory is given back under them.
    if (threadIdx.x == 0) set_status(p.status, sm.status.code, sm.status.detail);
    bool gone = false;
    if (warp == 8) {
      for (int i = max(0, sm.loads[0] - kKSlots); i < sm.loads[0]; ++i)
        if (2 * i != c.withhold) dwait_warp(&sm.k_full[i % kKSlots], (i / kKSlots) & 1, p.status, 92, gone);
      for (int i = max(0, sm.loads[1] - kVSlots); i < sm.loads[1]; ++i)
        if (2 * i + 1 != c.withhold) dwait_warp(&sm.v_full[i % kVSlots], (i / kVSlots) & 1, p.status, 92, gone);
      for (int x = 0; x < 2; ++x)
        if (sm.loads[2 + x] > 0) dwait_warp(&sm.q_full[x], (sm.loads[2 + x] - 1) & 1, p.status, 92, gone);
    } else if (warp == 9) {
      umma_commit_lead(elect_one(), &sm.drain);
      dwait_warp(&sm.drain, 0, p.status, 93, gone);
    }
    __syncthreads();
  }
  if (warp == 9) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

}  // namespace

void launch_window_prompt(const WindowPromptParams& c, int grid, cudaStream_t st) {
  static std::once_flag once;
  std::call_once(once, [] {
    cudaFuncSetAttribute(window_prompt_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(PromptSmem) + 1024);
  });
  window_prompt_kernel<<<grid, kThreads, sizeof(PromptSmem) + 1024, st>>>(c);
  count_launch();
  if (c.p.splits > 1) launch_window_join(c.p, st);
}

}  // namespace uc
