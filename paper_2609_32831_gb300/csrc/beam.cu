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
// 1. beam_tile_kernel: one CTA per tile of kBeamTile logits of a row, which
//    stay in registers: their maximum, the sum of exp(x - max) and the tile's
//    best n logits. The logits are read once.
// 2. beam_merge_kernel: one CTA per request joins its tiles.
#include "common.cuh"
#include "internal.h"

namespace uc {

namespace {

constexpr int kSelThreads = 256;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kPer = kBeamTile / kSelThreads;  // logits per thread
constexpr int kSelGroups = 64;                 // thread groups whose maxima bound the n-th best
constexpr int kGroupLanes = kSelThreads / kSelGroups;
static_assert(kSelGroups >= UC_MAX_BEAM_OUT, "n groups have to exist");
// The n-th largest of the groups' maxima is at most the tile's n-th largest
// logit, and only n groups reach it: no more candidates than their logits.
constexpr int kSelCap = UC_MAX_BEAM_OUT * kGroupLanes * kPer;
constexpr float kNegInf = -INFINITY;
constexpr float kLog2e = 1.4426950408889634f;

// Order-preserving map of floats (no NaN) to unsigned integers; -0 and +0 map
// to one value.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
// (logit, position) as one key: the higher logit, then the lower position.
__device__ __forceinline__ uint64_t logit_key(float x, uint32_t pos) {
  return ((uint64_t)ordered(x) << 32) | (0xffffffffu - pos);
}

template <typename T>
__device__ __forceinline__ float to_float(T x);
template <>
__device__ __forceinline__ float to_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <>
__device__ __forceinline__ float to_float<__half>(__half x) { return __half2float(x); }
// A logit as the selection sees it: NaN and +inf (reported as UC_ERR_RANGE)
// count as -inf, so that every bound below holds for them too.
template <typename T>
__device__ __forceinline__ float logit(T x) {
  const float f = to_float(x);
  return f < INFINITY ? f : kNegInf;
}

__device__ __forceinline__ uint64_t shfl_xor_u64(uint64_t x, int m) {
  const uint32_t lo = __shfl_xor_sync(0xffffffffu, (uint32_t)x, m);
  const uint32_t hi = __shfl_xor_sync(0xffffffffu, (uint32_t)(x >> 32), m);
  return ((uint64_t)hi << 32) | lo;
}

// A finished beam goes on with the end token alone, at no cost: as if its
// logits were 0 there and -inf elsewhere. Writes the tile's part of that.
__device__ void finished_tile(const BeamParams& p, int row, int tile, int len) {
  const int lo = tile * kBeamTile;
  const bool here = p.eos >= lo && p.eos < lo + len;
  const size_t at = (size_t)row * p.tiles + tile;
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

template <typename T>
__global__ void __launch_bounds__(kSelThreads) beam_tile_kernel(const __grid_constant__ BeamParams p) {
  __shared__ uint64_t s_group[kSelGroups];
  __shared__ float s_red[kSelWarps];
  __shared__ uint16_t s_cand[kSelCap];
  __shared__ int s_count, s_bad;
  __shared__ uint64_t s_tau;
  griddep_launch_dependents();
  const int tile = blockIdx.x, row = blockIdx.y;
  const int b = row / p.beams, kb = row % p.beams;
  const int lo = tile * kBeamTile, len = min(kBeamTile, p.vocab - lo);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (p.finished != nullptr && p.finished[row]) {
    finished_tile(p, row, tile, len);
    return;
  }
  if (threadIdx.x == 0) {
    s_count = 0;
    s_bad = 0;
  }
  const T* x = static_cast<const T*>(p.logits) + b * p.stride_b + kb * p.stride_k + lo;
  // thread t holds logits t, t + 256, ...
  float v[kPer];
  float best = kNegInf;
  int best_at = threadIdx.x;
  bool bad = false;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int i = e * kSelThreads + threadIdx.x;
    v[e] = kNegInf;
    if (i < len) {
      v[e] = logit(x[i]);
      bad |= !(to_float(x[i]) < INFINITY);
    }
    if (v[e] > best) {
      best = v[e];
      best_at = i;
    }
  }
  float m = best;
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) s_red[warp] = m;
  uint64_t key = logit_key(best, best_at);
#pragma unroll
  for (int o = 1; o < kGroupLanes; o <<= 1) {
    const uint64_t other = shfl_xor_u64(key, o);
    key = key > other ? key : other;
  }
  if (threadIdx.x % kGroupLanes == 0) s_group[threadIdx.x / kGroupLanes] = key;
  __syncthreads();
  if (bad) s_bad = 1;
#pragma unroll
  for (int w = 0; w < kSelWarps; ++w) m = fmaxf(m, s_red[w]);
  // the n-th largest group maximum (positions differ, so keys do)
  const int n = min(p.n, len);
  if (threadIdx.x < kSelGroups) {
    const uint64_t mine = s_group[threadIdx.x];
    int rank = 0;
    for (int g = 0; g < kSelGroups; ++g) rank += s_group[g] > mine;
    if (rank == n - 1) s_tau = mine;
  }
  const float base = m == kNegInf ? 0.f : m;
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < kPer; ++e) sum += ex2_approx((v[e] - base) * kLog2e);
#pragma unroll
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  __syncthreads();
  if (lane == 0) s_red[warp] = sum;
  const uint64_t tau = s_tau;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int i = e * kSelThreads + threadIdx.x;
    if (i < len && logit_key(v[e], i) >= tau) s_cand[atomicAdd(&s_count, 1)] = (uint16_t)i;
  }
  __syncthreads();
  const size_t at = (size_t)row * p.tiles + tile;
  if (threadIdx.x == 0) {
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < kSelWarps; ++w) total += s_red[w];
    p.part_ms[at] = make_float2(m, total);
    if (s_bad) set_status(p.status, UC_ERR_RANGE, row);
  }
  // the candidates' ranks; the first n are the tile's best
  const int c = s_count;
  for (int i = threadIdx.x; i < c; i += kSelThreads) {
    const int pos = s_cand[i];
    const float xi = logit(x[pos]);
    const uint64_t mine = logit_key(xi, pos);
    int rank = 0;
    for (int j = 0; j < c && rank < n; ++j) rank += logit_key(logit(x[s_cand[j]]), s_cand[j]) > mine;
    if (rank < n) {
      p.part_x[at * p.n + rank] = xi;
      p.part_tok[at * p.n + rank] = lo + pos;
    }
  }
  for (int i = n + threadIdx.x; i < p.n; i += kSelThreads) {
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
  __shared__ CandKey s_tau, s_key[kMaxMerge];
  __shared__ int s_id[kMaxMerge];
  __shared__ int s_count;
  griddep_wait();
  const int b = blockIdx.x;
  const int lists = p.beams * p.tiles;
  if (threadIdx.x == 0) {
    s_count = 0;
    s_tau = CandKey{0, 0};
  }
  // each beam's log sum exp over its tiles, one warp per beam
  for (int kb = threadIdx.x >> 5; kb < p.beams; kb += kMergeThreads / 32) {
    const int lane = threadIdx.x & 31;
    const float2* ms = p.part_ms + ((size_t)b * p.beams + kb) * p.tiles;
    float m = kNegInf;
    for (int t = lane; t < p.tiles; t += 32) m = fmaxf(m, ms[t].x);
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float base = m == kNegInf ? 0.f : m;
    float sum = 0.f;
    for (int t = lane; t < p.tiles; t += 32)
      if (ms[t].x != kNegInf) sum += ms[t].y * expf(ms[t].x - base);
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) {
      const float sc = p.scores[(size_t)b * p.beams + kb];
      s_base[kb] = base;
      s_log[kb] = logf(sum);
      s_score[kb] = sc;
      if (!(sc < INFINITY)) set_status(p.status, UC_ERR_RANGE, b * p.beams + kb);
    }
  }
  __syncthreads();
  auto score_of = [&](int kb, float x) {
    return x == kNegInf ? kNegInf : s_score[kb] + ((x - s_base[kb]) - s_log[kb]);
  };
  const size_t first = (size_t)b * lists * p.n;
  auto key_of = [&](int id) {  // id: list * n + rank; a, b = 0 where there is no such candidate
    const int tok = p.part_tok[first + id];
    if (tok < 0) return CandKey{0, 0};
    const int kb = id / p.n / p.tiles;
    const float x = p.part_x[first + id];
    return CandKey{((uint64_t)ordered(score_of(kb, x)) << 32) | (0xffffffffu - kb), logit_key(x, tok)};
  };
  // the n-th best list head bounds the result from below, and only n lists
  // reach it
  const int n = p.n;
  if (lists > n)
    for (int l = threadIdx.x; l < lists; l += kMergeThreads) {
      const CandKey mine = key_of(l * n);
      int rank = 0;
      for (int o = 0; o < lists && rank < n; ++o) rank += key_of(o * n).before(mine);
      if (rank == n - 1) s_tau = mine;
    }
  __syncthreads();
  const CandKey tau = s_tau;
  for (int l = threadIdx.x; l < lists; l += kMergeThreads)
    for (int r = 0; r < n; ++r) {
      const CandKey k = key_of(l * n + r);
      if ((k.a | k.b) == 0 || tau.before(k)) break;
      const int at = atomicAdd(&s_count, 1);
      s_key[at] = k;
      s_id[at] = l * n + r;
    }
  __syncthreads();
  const int c = s_count;
  for (int i = threadIdx.x; i < c; i += kMergeThreads) {
    const CandKey mine = s_key[i];
    int rank = 0;
    for (int j = 0; j < c && rank < n; ++j) rank += s_key[j].before(mine);
    if (rank < n) {
      const int kb = s_id[i] / n / p.tiles;
      const int tok = p.part_tok[first + s_id[i]];
      const size_t o = (size_t)b * n + rank;
      p.out_scores[o] = score_of(kb, p.part_x[first + s_id[i]]);
      p.out_parent[o] = kb;
      p.out_token[o] = tok;
      if (p.out_finished)
        p.out_finished[o] = tok == p.eos || (p.finished != nullptr && p.finished[(size_t)b * p.beams + kb]);
    }
  }
}

// ---------------------------------------------------------------- reorder
// One work unit: kReorderBytes of one block of one array. Copies are 16 bytes
// wide where both blocks allow it, four bytes otherwise and at the end.
constexpr int kCopyThreads = 256;

__global__ void __launch_bounds__(kCopyThreads) reorder_kernel(const __grid_constant__ ReorderParams p) {
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
  reorder_kernel<<<p.n_units < 8 * num_sms() ? p.n_units : 8 * num_sms(), kCopyThreads, 0, st>>>(p);
  count_launch();
}

}  // namespace uc
