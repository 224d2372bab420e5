// Generation with several continuations (beams) per request: selection of the
// best continuations over a request's beams and vocabulary, and the
// reordering of caches and states that follows it.
//
// Selection. A continuation of beam b by token v scores
//   c = score_b + ((x_bv - m_b) - log sum_v exp(x_bv - m_b)),  m_b = max_v x_bv.
// The best n of a request come out in the order: higher score, lower beam,
// higher logit, lower token (a total order, so the result does not depend on
// how the work is split). Within a beam the score grows with the logit, so a
// row's best n logits are all that can be chosen.
// 1. beam_tile_kernel: one CTA per tile of a row, 2048 16-byte vectors at a
//    time in registers: their maximum, the sum of exp(x - max) and the tile's
//    best n logits. The logits are read once, the next vectors while these are
//    worked on.
//    The floor is HBM where rows are many: an SM's share is 11 two-byte logits
//    per cycle, the exponentials alone take 16 of the SM's per cycle at most.
//    256 rows of 150001 bf16 logits: 27 us, 2.9 TB/s; bound by dependent steps
//    between one barrier per round. (A kernel that ranked all thread maxima per
//    2048 vectors took 65 us; candidates listed per warp, with no barrier, let
//    twice as many through: 44 us; half the vectors per round and twice the
//    CTAs: the same.)
// 2. beam_merge_kernel: one CTA per request joins its tiles: about 8 us alone,
//    four loads one after the other; it starts while the tiles run.
#include <algorithm>

#include "common.cuh"
#include "internal.h"
#include "logits.cuh"
#include "tcgen05.cuh"

namespace uc {

namespace {

constexpr int kSelThreads = 256;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kVecs = 8;  // 16-byte vectors per thread and round
constexpr int kRound = kSelThreads * kVecs;
constexpr int kSelGroups = 64;  // groups of four threads
// Candidates: the n-th largest of a round's thread maxima is at most its n-th
// largest logit, and fewer than n threads hold larger ones; n equal ones; and
// what the rounds before left, fewer than many(n).
constexpr __host__ __device__ int many(int n) { return 2 * n + 16; }
constexpr int kSelCap = many(UC_MAX_BEAM_OUT) + UC_MAX_BEAM_OUT * kVecs * 8;
constexpr float kNegInf = -INFINITY;
static_assert(kSelGroups >= UC_MAX_BEAM_OUT, "n groups have to exist");

// Order-preserving map of floats (no NaN) to unsigned integers; -0 and +0 map
// to one value.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}
// (logit, position) as one key: the higher logit, then the lower position.
__device__ __forceinline__ uint64_t logit_key(float x, uint32_t pos) {
  return ((uint64_t)ordered(x) << 32) | (0xffffffffu - pos);
}

// A finished beam goes on with the end token alone, at no cost: as if its
// logits were 0 there and -inf elsewhere. Writes the part of that of tokens lo
// .. lo + len - 1.
__device__ void finished_tile(const BeamParams& p, size_t at, int lo, int len) {
  const bool here = p.eos >= lo && p.eos < lo + len;
  if (threadIdx.x == 0) p.part_ms[at] = here ? make_float2(0.f, 1.f) : make_float2(kNegInf, 0.f);
  const int i = threadIdx.x;
  if (i < p.n) {
    // rank 0: the end token if it lies here; then the other tokens in order
    int tok = lo + i;
    float x = kNegInf;
    if (here) {
      if (i == 0) {
        tok = p.eos;
        x = 0.f;
      } else {
        tok = lo + i - 1 < p.eos ? lo + i - 1 : lo + i;
      }
    }
    p.part_x[at * p.n + i] = x;
    p.part_tok[at * p.n + i] = i < len ? tok : -1;
  }
}

// The k-th largest (from 1) of COUNT values, ties by place: the CTA's threads
// share each value's ranking out.
template <int COUNT>
__device__ __forceinline__ void kth_largest(const uint32_t* vals, int k, float* out) {
  constexpr int kPer = kSelThreads / COUNT;  // threads per value
  const int g = threadIdx.x / kPer, part = threadIdx.x % kPer * (COUNT / kPer);
  const uint32_t mine = vals[g];
  int rank = 0;
#pragma unroll 4
  for (int o = part; o < part + COUNT / kPer; o += 4) {
    const uint4 w = *reinterpret_cast<const uint4*>(vals + o);
    rank += (w.x > mine || (w.x == mine && o < g)) + (w.y > mine || (w.y == mine && o + 1 < g)) +
            (w.z > mine || (w.z == mine && o + 2 < g)) + (w.w > mine || (w.w == mine && o + 3 < g));
  }
#pragma unroll
  for (int o = 1; o < kPer; o <<= 1) rank += __shfl_xor_sync(0xffffffffu, rank, o);
  if (threadIdx.x % kPer == 0 && rank == k - 1) *out = unordered(mine);
}

// The best n of c candidates, in order, to out(rank, key); every thread calls it.
template <typename F>
__device__ __forceinline__ void best_of(const uint64_t* keys, int c, int n, F&& out) {
  for (int i = threadIdx.x; i < c; i += kSelThreads) {
    const uint64_t mine = keys[i];
    int rank = 0;
    int j = 0;
    for (; j + 8 <= c && rank < n; j += 8)
#pragma unroll
      for (int u = 0; u < 8; ++u) rank += keys[j + u] > mine;
    for (; j < c && rank < n; ++j) rank += keys[j] > mine;
    if (rank < n) out(rank, mine);
  }
}

template <typename T>
__global__ void __launch_bounds__(kSelThreads, kBeamPerSm) beam_tile_kernel(const __grid_constant__ BeamParams p) {
  using L = Logits<T>;
  constexpr int kE = L::kE;
  __shared__ __align__(16) uint32_t s_max[kSelThreads];
  __shared__ float s_red[2][kSelWarps];
  __shared__ int s_scan[kSelWarps];
  __shared__ uint64_t s_key[kSelCap], s_best[UC_MAX_BEAM_OUT];
  __shared__ float s_tau;
  __shared__ int s_new[3];  // candidates of a round, of rounds in turn: zeroed a barrier before their round
  griddep_launch_dependents();
  const int tile = blockIdx.x, row = blockIdx.y;
  const int b = row / p.beams, kb = row % p.beams;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const T* const x = static_cast<const T*>(p.logits) + b * p.stride_b + kb * p.stride_k;
  // vectors lie on 16-byte boundaries: the row's first may start before it
  const int lead = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
  const int vec0 = min(tile * p.span, (int)(((int64_t)p.vocab + lead + kE - 1) / kE));
  const int vec1 = (int)min((int64_t)vec0 + p.span, ((int64_t)p.vocab + lead + kE - 1) / kE);
  const int lo = max(0, (int)((int64_t)vec0 * kE - lead));
  const int len = max(0, (int)(min((int64_t)p.vocab, (int64_t)vec1 * kE - lead) - lo));
  const size_t at = (size_t)row * p.tiles + tile;
  if (p.finished != nullptr && p.finished[row]) {
    finished_tile(p, at, lo, len);
    return;
  }
  if (tid == 0) s_new[0] = 0;
  bool bad = false;
  const uint32_t vocab = (uint32_t)p.vocab;
  const uint4* const xv = reinterpret_cast<const uint4*>(x - lead);
  // vectors that the row has wholly
  const int whole0 = lead != 0, whole1 = min(vec1, (int)(((int64_t)p.vocab + lead) / kE));
  // round vectors from `from`: thread t holds vectors t, t + 256, ...
  auto token = [&](int vec, int e) { return (uint32_t)vec * kE + e - lead; };  // (not below vocab: no token)
  auto load = [&](uint4(&v)[kVecs], int from) {
    const uint4* const at = xv + from + tid;
    if (from >= whole0 && from + kRound <= whole1) {
#pragma unroll
      for (int k = 0; k < kVecs; ++k) v[k] = at[k * kSelThreads];
      return;
    }
    const uint32_t none = L::raw(kNegInf), fill = kE == 4 ? none : none | none << 16;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const int i = from + k * kSelThreads + tid;
      v[k] = make_uint4(fill, fill, fill, fill);
      if (i >= whole0 && i < whole1) v[k] = at[k * kSelThreads];
    }
  };
  uint4 v[kVecs], next[kVecs];
  float best_of_all = kNegInf, sum = 0.f, tau = kNegInf;
  const int n = min(p.n, len);
  int count = 0, turn = 0;  // candidates so far (equal in every thread)
  load(next, vec0);
  for (int from = vec0; from < vec1; from += kRound) {
    int* const fresh = s_new + turn;
    turn = turn == 2 ? 0 : turn + 1;
    if (tid == 0) s_new[turn] = 0;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) v[k] = next[k];
    if (from + kRound < vec1) load(next, from + kRound);
    // a row's ends: only what the row has
    if (from < whole0 || (whole1 < vec1 && from + kRound > whole1)) {
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        const int i = from + k * kSelThreads + tid;
        if (i < vec1 && (i < whole0 || i >= whole1))
          v[k] = make_vector<T>([&](int e) {
            const uint32_t t = token(i, e);
            const float f = to_float(x[min(t, vocab - 1)]);  // (loads that wait for nothing)
            return t < vocab ? f : kNegInf;
          });
      }
    }
    float best = kNegInf;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const float m = L::largest(v[k]);
      asm("max.NaN.f32 %0, %0, %1;" : "+f"(best) : "f"(m));
    }
    if (!(best < INFINITY)) {
      // NaN or +inf, reported as UC_ERR_RANGE: they count as -inf
      bad = true;
      best = kNegInf;
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        v[k] = make_vector<T>([&](int e) {
          const float f = L::get(v[k], e);
          return f < INFINITY ? f : kNegInf;
        });
        best = fmaxf(best, L::largest(v[k]));
      }
    }
    if (from == vec0) {  // a bound on the tile's n-th largest: that of the first round's groups
      float m = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, 1));
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
      if ((lane & 3) == 0) s_max[tid >> 2] = ordered(m);
      __syncthreads();
      kth_largest<kSelGroups>(s_max, n, &s_tau);
    }
    // the candidates: everything from tau up in the first round, which has n
    // of them; above tau after it, where equal ones come too late
    bool more = best > tau;
    if (from == vec0) {
      __syncthreads();
      tau = s_tau;
      more = best >= tau;
    }
    const int before = count;
    auto take = [&](bool equal) {  // its logits above tau or equal to it, as far as there is room
      uint32_t mask = 0;
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        const float m = L::largest(v[k]);
        mask |= (uint32_t)(m > tau || (equal && m == tau)) << k;
      }
      for (; mask; mask &= mask - 1) {
        const int k = __ffs(mask) - 1, i = from + k * kSelThreads + tid;
        uint4 w = v[0];
#pragma unroll
        for (int j = 1; j < kVecs; ++j)
          if (j == k) w = v[j];
        uint32_t hits = 0;
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          const float f = L::get(w, e);
          hits |= (uint32_t)(f > tau || (equal && f == tau)) << e;
        }
        for (; hits; hits &= hits - 1) {
          const int e = __ffs(hits) - 1;
          if (i >= vec1 || token(i, e) >= vocab) continue;  // what fills the last vectors up
          const int c = before + atomicAdd(fresh, 1);
          if (c < kSelCap) s_key[c] = logit_key(L::get(w, e), token(i, e));
        }
      }
    };
    if (more) take(from == vec0);
    // sum of exp(x - m) with m the thread's maximum so far. The difference is
    // taken before it is scaled: it is at most 0, so no finite logits overflow
    // (a mask of the type's lowest value, a thread that holds nothing else), and
    // its rounding is 2^-24 of itself
    const float top = fmaxf(best_of_all, best), base = top == kNegInf ? 0.f : top;
    const uint64_t l2 = f2_pack(kLog2e, kLog2e), nb = f2_pack(-base, -base);
    uint64_t acc[2] = {0ull, 0ull};
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      if (from + k * kSelThreads >= vec1) break;
#pragma unroll
      for (int e = 0; e < kE; e += 2) {
        float a, c;
        f2_unpack(f2_mul(f2_add(f2_pack(L::get(v[k], e), L::get(v[k], e + 1)), nb), l2), a, c);
        acc[(e >> 1) & 1] = f2_add(acc[(e >> 1) & 1], f2_pack(ex2_approx(a), ex2_approx(c)));
      }
    }
    float part[4];
    f2_unpack(acc[0], part[0], part[1]);
    f2_unpack(acc[1], part[2], part[3]);
    sum = fmaf(sum, ex2_approx((best_of_all - base) * kLog2e), (part[0] + part[1]) + (part[2] + part[3]));
    best_of_all = top;
    __syncthreads();
    count = before + *fresh;
    if (count > kSelCap) {
      // many large or many equal ones: bounded closer by this round's threads'
      // maxima, with equal ones by place until the round has n
      s_max[tid] = ordered(best);
      __syncthreads();
      kth_largest<kSelThreads>(s_max, min(n, kSelThreads), &s_tau);
      if (tid == 0) *fresh = 0;
      __syncthreads();
      tau = fmaxf(tau, s_tau);
      take(false);
      __syncthreads();
      int want = n - *fresh;
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        if (want <= 0) break;
        const int i = from + k * kSelThreads + tid;
        uint32_t mask = 0;
#pragma unroll
        for (int e = 0; e < kE; ++e)
          mask |= (uint32_t)(i < vec1 && token(i, e) < vocab && L::get(v[k], e) == tau) << e;
        int ahead = __popc(mask);
        const int mine = ahead;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, ahead, o);
          if (lane >= o) ahead += y;
        }
        __syncthreads();
        if (lane == 31) s_scan[warp] = ahead;
        __syncthreads();
        ahead -= mine;
        int total = 0;
        for (int w = 0; w < kSelWarps; ++w) {
          if (w < warp) ahead += s_scan[w];
          total += s_scan[w];
        }
        for (; mask && ahead < want; mask &= mask - 1, ++ahead)
          s_key[before + atomicAdd(fresh, 1)] = logit_key(tau, token(i, __ffs(mask) - 1));
        want -= total;
      }
      __syncthreads();
      count = before + *fresh;
    }
    if (count > many(n) && from + kRound < vec1) {
      best_of(s_key, count, n, [&](int rank, uint64_t key) { s_best[rank] = key; });
      __syncthreads();
      if (tid < n) s_key[tid] = s_best[tid];
      count = n;
      tau = unordered((uint32_t)(s_best[n - 1] >> 32));
      __syncthreads();
    }
  }
  // the tile's maximum and sum
  float m = best_of_all;
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) s_red[0][warp] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSelWarps; ++w) m = fmaxf(m, s_red[0][w]);
  if (m != kNegInf) sum *= ex2_approx((best_of_all - m) * kLog2e);
#pragma unroll
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s_red[1][warp] = sum;
  bad = __syncthreads_or(bad);
  if (tid == 0) {
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < kSelWarps; ++w) total += s_red[1][w];
    p.part_ms[at] = make_float2(m, total);
    if (bad) set_status(p.status, UC_ERR_RANGE, row);
  }
  best_of(s_key, count, n, [&](int rank, uint64_t key) {
    p.part_x[at * p.n + rank] = unordered((uint32_t)(key >> 32));
    p.part_tok[at * p.n + rank] = (int32_t)(0xffffffffu - (uint32_t)key);
  });
  for (int i = n + tid; i < p.n; i += kSelThreads) {
    p.part_x[at * p.n + i] = kNegInf;
    p.part_tok[at * p.n + i] = -1;  // no such candidate
  }
}

// A candidate's place in the result's order as two words.
struct CandKey {
  uint64_t a, b;
  __device__ __forceinline__ bool before(const CandKey& o) const { return a != o.a ? a > o.a : b > o.b; }
};

constexpr int kMergeThreads = 256;
constexpr int kMaxMerge = UC_MAX_BEAM_OUT * UC_MAX_BEAM_OUT;  // n lists of n candidates

__global__ void __launch_bounds__(kMergeThreads) beam_merge_kernel(const __grid_constant__ BeamParams p) {
  __shared__ float s_base[UC_MAX_BEAMS], s_log[UC_MAX_BEAMS], s_score[UC_MAX_BEAMS];
  __shared__ CandKey s_tau, s_key[kMaxMerge], s_head[kBeamLists];
  __shared__ int s_id[kMaxMerge], s_list[UC_MAX_BEAM_OUT];
  __shared__ int s_count, s_lists;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31;
  const int lists = p.beams * p.tiles, n = p.n;
  if (tid == 0) {
    s_count = 0;
    s_lists = 0;
    s_tau = CandKey{0, 0};
  }
  griddep_wait();
  const size_t row0 = (size_t)b * p.beams, first = (size_t)b * lists * n;
  // each beam's log sum exp over its tiles, one warp per beam
  for (int kb = tid >> 5; kb < p.beams; kb += kMergeThreads / 32) {
    const float2* ms = p.part_ms + (row0 + kb) * p.tiles;
    float m = kNegInf, sum = 0.f;
    for (int t = lane; t < p.tiles; t += 32) {
      const float2 x = ms[t];
      if (x.x > m) {
        sum = fmaf(sum, expf(m - x.x), x.y);
        m = x.x;
      } else if (x.x != kNegInf) {
        sum = fmaf(x.y, expf(x.x - m), sum);
      }
    }
    float top = m;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float base = top == kNegInf ? 0.f : top;
    if (m != kNegInf) sum *= expf(m - base);
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) {
      const float sc = p.scores[row0 + kb];
      s_base[kb] = base;
      s_log[kb] = logf(sum);
      s_score[kb] = sc;
      if (!(sc < INFINITY)) set_status(p.status, UC_ERR_RANGE, (int)(row0 + kb));
    }
  }
  __syncthreads();
  auto score_of = [&](int kb, float x) {
    return x == kNegInf ? kNegInf : s_score[kb] + ((x - s_base[kb]) - s_log[kb]);
  };
  auto key_of = [&](int list, int r) {  // a, b = 0 where there is no such candidate
    const size_t id = first + (size_t)list * n + r;
    const int tok = p.part_tok[id];
    const float x = p.part_x[id];
    if (tok < 0) return CandKey{0, 0};
    const int kb = list / p.tiles;
    return CandKey{((uint64_t)ordered(score_of(kb, x)) << 32) | (0xffffffffu - kb), logit_key(x, tok)};
  };
  // the n-th best list head bounds the result from below, and only n lists
  // reach it
  for (int l = tid; l < lists; l += kMergeThreads) s_head[l] = key_of(l, 0);
  __syncthreads();
  if (lists > n) {
    for (int l = tid; l < lists; l += kMergeThreads) {
      const CandKey mine = s_head[l];
      int rank = 0;
#pragma unroll 8
      for (int o = 0; o < lists; ++o) rank += s_head[o].before(mine);
      if (rank == n - 1) s_tau = mine;  // (no two candidates are equal; where fewer exist, none is the n-th)
    }
    __syncthreads();
  }
  const CandKey tau = s_tau;
  for (int l = tid; l < lists; l += kMergeThreads) {
    const CandKey head = s_head[l];
    if ((head.a | head.b) != 0 && !tau.before(head)) s_list[atomicAdd(&s_lists, 1)] = l;
  }
  __syncthreads();
  for (int i = tid; i < s_lists * n; i += kMergeThreads) {
    const int l = s_list[i / n], r = i % n;
    const CandKey k = key_of(l, r);
    if ((k.a | k.b) == 0 || tau.before(k)) continue;
    const int at = atomicAdd(&s_count, 1);
    s_key[at] = k;
    s_id[at] = l;
  }
  __syncthreads();
  const int c = s_count;
  for (int i = tid; i < c; i += kMergeThreads) {
    const CandKey mine = s_key[i];
    int rank = 0;
#pragma unroll 4
    for (int j = 0; j < c; ++j) rank += s_key[j].before(mine);
    if (rank < n) {
      const int kb = s_id[i] / p.tiles;
      const int tok = (int)(0xffffffffu - (uint32_t)mine.b);
      const size_t o = (size_t)b * n + rank;
      p.out_scores[o] = score_of(kb, unordered((uint32_t)(mine.b >> 32)));
      p.out_parent[o] = kb;
      p.out_token[o] = tok;
      if (p.out_finished) p.out_finished[o] = tok == p.eos || (p.finished != nullptr && p.finished[row0 + kb]);
    }
  }
}

// ---------------------------------------------------------------- reorder
// One work unit: kReorderBytes of one block of one array. Copies are 16 bytes
// wide where both blocks allow it, four bytes otherwise and at the end. Bound
// by HBM: 281 MB read and as much written in 97 us, 5.8 TB/s.
constexpr int kCopyThreads = 256;

template <int N>
__global__ void __launch_bounds__(kCopyThreads) reorder_kernel(const __grid_constant__ ReorderParamsOf<N> p) {
  for (int u = blockIdx.x; u < p.n_units; u += gridDim.x) {
    int lo = 0, hi = p.n_arrays - 1;  // the array of this unit
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (p.a[mid].begin <= u) lo = mid; else hi = mid - 1;
    }
    const ReorderArray& a = p.a[lo];
    const int w = u - a.begin;
    const int part = w % a.parts, blk = w / a.parts;
    const int to = blk / a.heads, head = blk % a.heads;
    const int from = p.parent[to];
    if (from < 0 || from >= p.n_from) {
      if (threadIdx.x == 0) set_status(p.status, UC_ERR_RANGE, to);
      continue;
    }
    const int seq = to / p.n_to * p.n_from + from;
    int units = a.max_units;
    if (a.live != kLiveAll) {
      const int n = a.n_kept[seq];
      if (n < 0 || n > a.max_kept) {
        if (threadIdx.x == 0) set_status(p.status, UC_ERR_BUDGET, to);
        continue;
      }
      units = a.live == kLiveCount ? 1 : a.live == kLiveTokens ? n : a.live == kLiveGroups ? n / kGroup : n % kGroup;
    }
    const int64_t bytes = (int64_t)units * a.unit;
    const int64_t begin = (int64_t)part * kReorderBytes;
    const int64_t end = min(bytes, begin + kReorderBytes);
    if (begin >= end) continue;
    const uint8_t* src = a.src + ((int64_t)seq * a.heads + head) * a.src_block;
    uint8_t* dst = a.dst + ((int64_t)to * a.heads + head) * a.dst_block;
    int64_t done = begin;
    if (((reinterpret_cast<uintptr_t>(src) | reinterpret_cast<uintptr_t>(dst)) & 15) == 0) {
      const int64_t whole = end & ~int64_t(15);
      for (int64_t i = begin + 16 * threadIdx.x; i < whole; i += 16 * kCopyThreads)
        *reinterpret_cast<uint4*>(dst + i) = *reinterpret_cast<const uint4*>(src + i);
      done = max(begin, whole);
    }
    for (int64_t i = done + 4 * threadIdx.x; i < end; i += 4 * kCopyThreads)
      *reinterpret_cast<uint32_t*>(dst + i) = *reinterpret_cast<const uint32_t*>(src + i);
  }
}

}  // namespace

void launch_beam(const BeamParams& p, int dtype, cudaStream_t st) {
  const dim3 grid(p.tiles, p.batch * p.beams);
  if (dtype == UC_FP32)
    beam_tile_kernel<float><<<grid, kSelThreads, 0, st>>>(p);
  else if (dtype == UC_BF16)
    beam_tile_kernel<__nv_bfloat16><<<grid, kSelThreads, 0, st>>>(p);
  else
    beam_tile_kernel<__half><<<grid, kSelThreads, 0, st>>>(p);
  count_launch();
  launch_maybe_pdl(true, beam_merge_kernel, p.batch, kMergeThreads, 0, st, p);
  count_launch();
}

void launch_reorder(const ReorderParams& p, cudaStream_t st) {
  const int grid = p.n_units < 8 * num_sms() ? p.n_units : 8 * num_sms();
  if (p.n_arrays <= kReorderFew) {  // (18 KB of parameters are a good part of a small call's launch)
    ReorderParamsOf<kReorderFew> few;
    std::copy(p.a, p.a + p.n_arrays, few.a);
    few.parent = p.parent;
    few.status = p.status;
    few.n_arrays = p.n_arrays;
    few.n_seq = p.n_seq;
    few.n_from = p.n_from;
    few.n_to = p.n_to;
    few.n_units = p.n_units;
    reorder_kernel<kReorderFew><<<grid, kCopyThreads, 0, st>>>(few);
  } else {
    reorder_kernel<kReorderArrays><<<grid, kCopyThreads, 0, st>>>(p);
  }
  count_launch();
}

}  // namespace uc
