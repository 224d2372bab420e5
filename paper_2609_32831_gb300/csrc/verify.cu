// Verification of drafted tokens: which are accepted, and the token behind them.
//
// A draft d_t is accepted while u_t q_t(d_t) < p_t(d_t); the next token is the
// argmax of w_v / e_v with w = max(p_a - q_a, 0) behind a rejected draft and w = p_n
// behind the last (and where p_a - q_a leaves nothing but rounding). Softmax statistics need whole rows, the choice a second look at
// two of them:
// 1. verify_rows_kernel: one CTA per tile of a row (target's and drafter's): its
//    maximum and the sum of exp((x - max) / temperature), at temperature 0 the
//    maximum's place too.
// 2. verify_pick_kernel: every CTA joins the tiles of its sequence's rows, takes the
//    decisions, and looks through a part of the vocabulary for the next token; the
//    last CTA of a sequence writes its results.
// Bytes bound it where batches are large: all rows once (the second look finds
// them in L2). 32 sequences of five drafts, 150001 tokens, bf16: 33 us, of which the
// first kernel 20 (the rows' bytes 15.6), the second the noise's bytes and its own start; small
// batches 6 to 8 us, two kernels' latency.
#include <climits>
#include <cmath>
#include <cstring>

#include "args.h"
#include "common.cuh"
#include "internal.h"
#include "logits.cuh"
#include "tcgen05.cuh"

namespace uc {

namespace {

constexpr int kVerifyThreads = 256;
constexpr int kVerifyWarps = kVerifyThreads / 32;
constexpr int kVerifyVecs = 2;  // 16-byte vectors of a thread in flight, and as many worked on
constexpr int kRowsPerSm = 8;   // CTAs that an SM holds (with four of twice the vectors 22.6 us instead of 20)
constexpr int kPickPerSm = 4;
constexpr int kDeep = 8;         // tokens of a thread in flight
constexpr float kNone = -INFINITY;

__device__ __forceinline__ int drafts_of(const VerifyParams& p, int b) {
  return p.n_draft ? min(max(p.n_draft[b], 0), p.n_tok) : p.n_tok;
}
// 2^(d log2(e) / temperature), d <= 0
__device__ __forceinline__ float weight(const VerifyParams& p, float d) {
  d = fmaxf(d, -3e38f);  // (-inf times a remainder of 0 is not 0)
  return ex2_approx(fmaf(d, p.scale.x, d * p.scale.y));
}

template <typename T>
__device__ __forceinline__ const T* target_row(const VerifyParams& p, int b, int t) {
  return static_cast<const T*>(p.target) + b * p.target_b + t * p.target_t;
}
template <typename T>
__device__ __forceinline__ const T* draft_row(const VerifyParams& p, int b, int t) {
  return static_cast<const T*>(p.draft) + b * p.draft_b + t * p.draft_t;
}

// Rows are the target's [B, n_tok + 1], then the drafter's [B, n_tok].
template <typename T>
__global__ void __launch_bounds__(kVerifyThreads, kRowsPerSm) verify_rows_kernel(const __grid_constant__ VerifyParams p) {
  using L = Logits<T>;
  constexpr int kE = L::kE;
  __shared__ float s_m[kVerifyWarps], s_s[kVerifyWarps];
  __shared__ int s_at[kVerifyWarps];
  griddep_launch_dependents();
  const int tile = blockIdx.x % p.tiles, row = blockIdx.x / p.tiles;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int targets = p.batch * (p.n_tok + 1);
  const bool of_target = row < targets;
  const int b = of_target ? row / (p.n_tok + 1) : (row - targets) / p.n_tok;
  const int t = of_target ? row % (p.n_tok + 1) : (row - targets) % p.n_tok;
  if (of_target && t == 0 && tile == 0 && tid == 0) {
    p.best[b] = 0;
    p.done[b] = 0;
    if (p.n_draft && drafts_of(p, b) != p.n_draft[b]) set_status(p.status, UC_ERR_RANGE, b);
  }
  const int n = drafts_of(p, b);
  if (of_target ? t > n : t >= n) return;
  const T* const x = of_target ? target_row<T>(p, b, t) : draft_row<T>(p, b, t);
  // vectors lie on 16-byte boundaries: the row's first may start before it
  const int lead = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
  const int vecs = (int)(((int64_t)p.vocab + lead + kE - 1) / kE);
  const int vec0 = min(tile * p.span, vecs), vec1 = min(vec0 + p.span, vecs);
  const int whole0 = lead != 0, whole1 = (int)(((int64_t)p.vocab + lead) / kE);  // those the row has wholly
  const uint4* const xv = reinterpret_cast<const uint4*>(x - lead);
  float m = kNone, sum = 0.f;
  int at = INT_MAX;
  bool bad = false;
  constexpr int kRound = kVerifyThreads * kVerifyVecs;
  const int last = min(whole1, vec1);
  auto load = [&](uint4(&v)[kVerifyVecs], int from) {
    if (from - tid >= whole0 && from - tid + kRound <= last) {
#pragma unroll
      for (int k = 0; k < kVerifyVecs; ++k) v[k] = xv[from + k * kVerifyThreads];
      return;
    }
    // a row's ends: only what the row has
#pragma unroll
    for (int k = 0; k < kVerifyVecs; ++k) {
      const int i = from + k * kVerifyThreads;
      if (i >= whole0 && i < last) {
        v[k] = xv[i];
      } else {
        v[k] = make_vector<T>([&](int e) {
          const int64_t c = (int64_t)i * kE + e - lead;
          return i < vec1 && c >= 0 && c < p.vocab ? to_float(x[c]) : kNone;
        });
      }
    }
  };
  uint4 v[kVerifyVecs], next[kVerifyVecs];
  if (vec0 + tid < vec1) load(next, vec0 + tid);
  for (int from = vec0 + tid; from < vec1; from += kRound) {
#pragma unroll
    for (int k = 0; k < kVerifyVecs; ++k) v[k] = next[k];
    if (from + kRound < vec1) load(next, from + kRound);
    float best = kNone;
#pragma unroll
    for (int k = 0; k < kVerifyVecs; ++k) {
      const float largest = L::largest(v[k]);
      asm("max.NaN.f32 %0, %0, %1;" : "+f"(best) : "f"(largest));
    }
    if (!(best < INFINITY)) {
      // NaN or +inf, reported as UC_ERR_RANGE: they count as -inf
      bad = true;
      best = kNone;
#pragma unroll
      for (int k = 0; k < kVerifyVecs; ++k) {
        v[k] = make_vector<T>([&](int e) {
          const float f = L::get(v[k], e);
          return f < INFINITY ? f : kNone;
        });
        best = fmaxf(best, L::largest(v[k]));
      }
    }
    if (best > m) {
      sum *= weight(p, m - best);
      m = best;
      if (p.greedy) {
        at = INT_MAX;
#pragma unroll
        for (int k = 0; k < kVerifyVecs; ++k)
#pragma unroll
          for (int e = 0; e < kE; ++e)
            if (L::get(v[k], e) == best) at = min(at, (from + k * kVerifyThreads) * kE + e - lead);
      }
    }
    // the difference to the largest first: at most 0, whatever the logits' size
    const float base = m == kNone ? 0.f : m;
    const uint64_t nb = f2_pack(-base, -base), hi = f2_pack(p.scale.x, p.scale.x);
    uint64_t acc[2] = {0ull, 0ull};
#pragma unroll
    for (int k = 0; k < kVerifyVecs; ++k)
#pragma unroll
      for (int e = 0; e < kE; e += 2) {
        float c, d;
        f2_unpack(f2_mul(f2_add(f2_pack(L::get(v[k], e), L::get(v[k], e + 1)), nb), hi), c, d);
        acc[(e >> 1) & 1] = f2_add(acc[(e >> 1) & 1], f2_pack(ex2_approx(c), ex2_approx(d)));
      }
    float part[4];
    f2_unpack(acc[0], part[0], part[1]);
    f2_unpack(acc[1], part[2], part[3]);
    sum += (part[0] + part[1]) + (part[2] + part[3]);
  }
  float top = m;
#pragma unroll
  for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  if (m != top) at = INT_MAX;
  sum = m == kNone ? 0.f : sum * weight(p, m - top);
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    sum += __shfl_xor_sync(0xffffffffu, sum, d);
    at = min(at, __shfl_xor_sync(0xffffffffu, at, d));
  }
  if (lane == 0) {
    s_m[warp] = top;
    s_s[warp] = sum;
    s_at[warp] = at;
  }
  bad = __syncthreads_or(bad);
  if (tid == 0) {
    float tm = kNone, ts = 0.f;
    int ta = INT_MAX;
    for (int w = 0; w < kVerifyWarps; ++w) tm = fmaxf(tm, s_m[w]);
    for (int w = 0; w < kVerifyWarps; ++w) {
      if (s_m[w] != kNone) ts += s_s[w] * weight(p, s_m[w] - tm);
      if (s_m[w] == tm) ta = min(ta, s_at[w]);
    }
    const size_t to = (size_t)row * p.tiles + tile;
    p.part_ms[to] = make_float2(tm, ts);
    p.part_at[to] = ta;
    if (bad) set_status(p.status, UC_ERR_RANGE, b);
  }
}

template <typename T>
__global__ void __launch_bounds__(kVerifyThreads, kPickPerSm) verify_pick_kernel(const __grid_constant__ VerifyParams p) {
  __shared__ float s_m[2][UC_MAX_DRAFTS + 1], s_s[2][UC_MAX_DRAFTS + 1];
  __shared__ int s_at[UC_MAX_DRAFTS + 1], s_bad[2];
  __shared__ int s_a, s_last;
  __shared__ uint64_t s_key[kVerifyWarps];
  const int tile = blockIdx.x % p.pick_tiles, b = blockIdx.x / p.pick_tiles;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n = drafts_of(p, b), targets = p.batch * (p.n_tok + 1);
  const bool model = p.draft != nullptr;
  // what the caller gave is read while the rows are still at work: a draft's logits, the first noise
  int drafted = -1;
  float xd = kNone, yd = kNone, ud = 0.f, es[kDeep];
  if (tid < n) {
    drafted = p.tokens[b * p.n_tok + tid];
    if (drafted >= 0 && drafted < p.vocab && !p.greedy) {
      xd = to_float(target_row<T>(p, b, tid)[drafted]);
      if (model) yd = to_float(draft_row<T>(p, b, tid)[drafted]);
      ud = p.u[b * p.n_tok + tid];
    }
  }
  const int v_first = tile * p.pick_span + tid;
  const float* const noise = p.noise + (int64_t)b * p.vocab;
#pragma unroll
  for (int k = 0; k < kDeep; ++k) es[k] = p.greedy ? 1.f : noise[min(v_first + k * kVerifyThreads, p.vocab - 1)];
  griddep_wait();
  if (tid == 0) s_a = n;
  if (tid < 2) s_bad[tid] = 0;
  // the rows' statistics: a warp per row
  for (int i = warp; i < n + 1 + (model ? n : 0); i += kVerifyWarps) {
    const int which = i > n, t = which ? i - n - 1 : i;
    const int row = which ? targets + b * p.n_tok + t : b * (p.n_tok + 1) + t;
    const float2* const ms = p.part_ms + (size_t)row * p.tiles;
    float m = kNone, s = 0.f;
    int at = INT_MAX;
    for (int k = lane; k < p.tiles; k += 32) {
      const float2 x = ms[k];
      if (x.x > m) {
        s *= weight(p, m - x.x);
        m = x.x;
        at = INT_MAX;
      }
      if (x.x != kNone) s += x.y * weight(p, x.x - m);
      if (p.greedy && x.x == m) at = min(at, p.part_at[(size_t)row * p.tiles + k]);
    }
    float top = m;
#pragma unroll
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    if (m != top) at = INT_MAX;
    s = m == kNone ? 0.f : s * weight(p, m - top);
#pragma unroll
    for (int d = 16; d; d >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, d);
      at = min(at, __shfl_xor_sync(0xffffffffu, at, d));
    }
    if (lane == 0) {
      s_m[which][t] = top;
      s_s[which][t] = s;
      if (!which) s_at[t] = top == kNone ? 0 : at;
    }
  }
  __syncthreads();
  // log p of a token of row t of the target
  auto log_p = [&](int t, int v) {
    const float x = to_float(target_row<T>(p, b, t)[v]);
    return x < INFINITY && s_m[0][t] != kNone ? (x - s_m[0][t]) * p.inv_temperature - logf(s_s[0][t]) : kNone;
  };
  // the decisions: a thread per draft
  if (tid <= n) {
    const int t = tid;
    if (s_m[0][t] == kNone || (model && t < n && s_m[1][t] == kNone)) s_bad[0] = 1;
    bool good = drafted >= 0 && drafted < p.vocab;
    if (t < n && !good) s_bad[1] = 1;
    if (p.greedy) {
      good = good && s_m[0][t] != kNone && drafted == s_at[t];
    } else if (t < n) {
      // u q < p, with both sides times the two sums
      const float px = xd < INFINITY && s_m[0][t] != kNone ? weight(p, xd - s_m[0][t]) : 0.f;
      const float q = !model ? 1.f : yd < INFINITY && s_m[1][t] != kNone ? weight(p, yd - s_m[1][t]) : 0.f;
      good = good && ud * (q * s_s[0][t]) < px * (model ? s_s[1][t] : 1.f);
    }
    if (t < n && !good) atomicMin(&s_a, t);
  }
  __syncthreads();
  const int a = s_a;
  // the next token
  uint64_t key = 0;
  if (p.greedy) {
    key = 0xffffffffu - (uint32_t)s_at[a];
  } else {
    const T* const x = target_row<T>(p, b, a);
    const bool rest = a < n;
    const T* const y = model && rest ? draft_row<T>(p, b, a) : x;
    const float pm = s_m[0][a], ps = 1.f / s_s[0][a];
    const float qm = model && rest ? s_m[1][a] : 0.f, qs = model && rest ? 1.f / s_s[1][a] : 0.f;
    const int taken = !model && rest ? p.tokens[b * p.n_tok + a] : -1;
    const int v1 = min(p.vocab, (tile + 1) * p.pick_span);
    constexpr float kKnown = 0x1p-20f;  // what p and q are known to, at least
    float best = 0.f;
    int best_at = v_first;
    for (int v0 = v_first; v0 < v1; v0 += kVerifyThreads * kDeep) {
      float xs[kDeep], ys[kDeep];
#pragma unroll
      for (int k = 0; k < kDeep; ++k) {
        const int w = min(v0 + k * kVerifyThreads, p.vocab - 1);
        xs[k] = to_float(x[w]);
        ys[k] = model && rest ? to_float(y[w]) : kNone;
        if (v0 != v_first) es[k] = noise[w];
      }
#pragma unroll
      for (int k = 0; k < kDeep; ++k) {
        const int v = v0 + k * kVerifyThreads;
        // (as the sums were formed; a difference above 0 is that of +inf)
        const float dx = xs[k] - pm, dy = ys[k] - qm;
        const float own = dx <= 0.f ? ex2_approx(dx * p.scale.x) * ps : 0.f;
        float w = own;
        if (dy <= 0.f) w = fmaf(ex2_approx(dy * p.scale.x), -qs, w);
        if (v == taken) w -= 1.f;
        w = __fdividef(w > kKnown * own ? w : 0.f, es[k]);
        if (v < v1 && w > best) {  // (the first of equal ones: v ascends; a noise of 0 or NaN: none)
          best = w;
          best_at = v;
        }
      }
    }
    // A weight's rank: its bits, the top one set. A CTA that has found nothing left of p - q
    // gives p's own best instead, without that bit: it counts where none has found any.
    uint32_t top_bit = 0x80000000u;
    if (!__syncthreads_or(best > 0.f)) {
      top_bit = 0u;
#pragma unroll 1
      for (int v = v_first; v < v1; v += kVerifyThreads) {
        const float dx = to_float(x[v]) - pm;
        const float w = dx <= 0.f ? __fdividef(ex2_approx(dx * p.scale.x) * ps, noise[v]) : 0.f;
        if (w > best) {
          best = w;
          best_at = v;
        }
      }
    }
    const uint32_t rank = __float_as_uint(best) | (best > 0.f ? top_bit : 0u);
    if (v_first < v1) key = ((uint64_t)rank << 32) | (0xffffffffu - (uint32_t)best_at);
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    const uint64_t other = __shfl_xor_sync(0xffffffffu, key, d);
    key = other > key ? other : key;
  }
  if (lane == 0) s_key[warp] = key;
  __syncthreads();
  if (tid == 0) {
    for (int w = 0; w < kVerifyWarps; ++w) key = s_key[w] > key ? s_key[w] : key;
    bool last = true;
    if (p.pick_tiles > 1) {
      atomicMax(reinterpret_cast<unsigned long long*>(&p.best[b]), (unsigned long long)key);
      __threadfence();
      last = atomicAdd(&p.done[b], 1) == p.pick_tiles - 1;
      __threadfence();
      if (last) key = atomicMax(reinterpret_cast<unsigned long long*>(&p.best[b]), 0ull);
    }
    s_last = last ? (int)(0xffffffffu - (uint32_t)key) : -1;
    if (last) {
      p.accepted[b] = a;
      if (s_bad[0] | s_bad[1]) set_status(p.status, UC_ERR_RANGE, b);
    }
  }
  __syncthreads();
  const int last = s_last;
  if (last < 0) return;
  for (int t = tid; t <= p.n_tok; t += kVerifyThreads) {
    const int v = t < a ? p.tokens[b * p.n_tok + t] : last;
    p.out_tokens[b * (p.n_tok + 1) + t] = t <= a ? v : -1;
    p.logprob[b * (p.n_tok + 1) + t] = t <= a ? log_p(t, v) : 0.f;
  }
}

template <typename T>
void launch_typed(const VerifyParams& p, cudaStream_t st) {
  const int64_t rows = (int64_t)p.batch * (p.n_tok + 1 + (p.draft ? p.n_tok : 0));
  verify_rows_kernel<T><<<(unsigned)(rows * p.tiles), kVerifyThreads, 0, st>>>(p);
  count_launch();
  launch_maybe_pdl(true, verify_pick_kernel<T>, dim3((unsigned)(p.batch * p.pick_tiles)), dim3(kVerifyThreads), 0, st, p);
  count_launch();
}

int64_t row_vecs(int32_t vocab, int element) {
  const int per = 16 / element;
  return ((int64_t)vocab + (per - 1) + (per - 1)) / per;
}
constexpr int kMostTiles = 64;
constexpr int kMinSpan = 512;       // vectors of a tile, where the row has them
constexpr int kPickMost = 256;      // parts of a vocabulary
constexpr int kPickMinSpan = 512;   // tokens of one

size_t verify_bytes(int64_t rows, int batch, int tiles) {
  return 256 + rows * tiles * (sizeof(float2) + sizeof(int32_t)) + batch * (sizeof(uint64_t) + sizeof(int32_t)) + 16;
}

}  // namespace

void launch_verify(const VerifyParams& p, int dtype, cudaStream_t st) {
  if (dtype == UC_FP32)
    launch_typed<float>(p, st);
  else if (dtype == UC_BF16)
    launch_typed<__nv_bfloat16>(p, st);
  else
    launch_typed<__half>(p, st);
}

}  // namespace uc

using namespace uc;

extern "C" {

size_t uc_verify_workspace_size(int32_t batch, int32_t n_tok, int32_t vocab) {
  UC_TRACE();
  if (batch < 1 || n_tok < 1 || vocab < 1) return 0;
  return verify_bytes((int64_t)batch * (2 * (int64_t)n_tok + 1), batch,
                      (int)std::min<int64_t>(kMostTiles, (row_vecs(vocab, 4) + kMinSpan - 1) / kMinSpan));
}

uc_status uc_verify_draft(const void* target, int64_t target_b, int64_t target_t, const void* draft, int64_t draft_b,
                          int64_t draft_t, int32_t dtype, int32_t batch, int32_t n_tok, int32_t vocab,
                          const int32_t* tokens, const int32_t* n_draft, const float* u, const float* noise,
                          double temperature, int32_t* accepted, int32_t* out_tokens, float* logprob, void* workspace,
                          size_t workspace_bytes, void* stream) {
  UC_TRACE();
  const char* const fn = "uc_verify_draft";
  if (dtype != UC_FP32 && dtype != UC_BF16 && dtype != UC_FP16) {
    set_error("uc_verify_draft: bad logits type %d", dtype);
    return UC_ERR_ARG;
  }
  if (batch < 1 || n_tok < 1 || n_tok > UC_MAX_DRAFTS || vocab < 1 || vocab > (1 << 30) ||
      (int64_t)batch * (n_tok + 1) > 65535) {
    set_error("uc_verify_draft: unsupported shape (batch %d, drafts %d, vocabulary %d)", batch, n_tok, vocab);
    return UC_ERR_SHAPE;
  }
  const bool greedy = temperature == 0.0;
  if (greedy) draft = nullptr;
  constexpr int64_t kFar = int64_t(1) << 40;
  if (target_t < vocab || target_t > kFar || (batch > 1 && (target_b < 1 || target_b > kFar)) ||
      (draft != nullptr && ((n_tok > 1 && (draft_t < vocab || draft_t > kFar)) ||
                            (batch > 1 && (draft_b < 1 || draft_b > kFar))))) {
    set_error("uc_verify_draft: rows overlap or lie too far apart (strides %lld, %lld and %lld, %lld)", (long long)target_b,
              (long long)target_t, (long long)draft_b, (long long)draft_t);
    return UC_ERR_SHAPE;
  }
  if (!std::isfinite(temperature) || temperature < 0.0 || (!greedy && !(temperature >= 1e-6 && temperature <= 1e6))) {
    set_error("uc_verify_draft: temperature %g is neither 0 nor from 1e-6 to 1e6", temperature);
    return UC_ERR_ARG;
  }
  const int element = dtype == UC_FP32 ? 4 : 2;
  if (target == nullptr || tokens == nullptr || accepted == nullptr || out_tokens == nullptr || logprob == nullptr ||
      (!greedy && (u == nullptr || noise == nullptr)) || !aligned(target, element) || !aligned(draft, element) ||
      !aligned(tokens, 4) || !aligned(n_draft, 4) || !aligned(u, 4) || !aligned(noise, 4) || !aligned(accepted, 4) ||
      !aligned(out_tokens, 4) || !aligned(logprob, 4)) {
    set_error("uc_verify_draft: null or misaligned argument");
    return UC_ERR_ARG;
  }
  const uc_status st = check_workspace(workspace, workspace_bytes, uc_verify_workspace_size(batch, n_tok, vocab), fn);
  if (st != UC_OK) return st;
  if (batch == 1) target_b = draft_b = 0;
  if (n_tok == 1) draft_t = 0;
  auto extent = [&](int64_t sb, int64_t st, int n) { return (uint64_t)element * ((batch - 1) * sb + (n - 1) * st + vocab); };
  const uint64_t bt = 4ull * batch * n_tok;
  struct { const void* p; uint64_t bytes; } out[3] = {{accepted, 4ull * batch}, {out_tokens, bt + 4ull * batch},
                                                      {logprob, bt + 4ull * batch}},
      in[6] = {{target, extent(target_b, target_t, n_tok + 1)},
               {draft, draft ? extent(draft_b, draft_t, n_tok) : 0},
               {tokens, bt},
               {n_draft, n_draft ? 4ull * batch : 0},
               {u, greedy ? 0 : bt},
               {noise, greedy ? 0 : 4ull * batch * vocab}};
  for (int i = 0; i < 3; ++i) {
    bool shared = false;
    for (const auto& x : in) shared |= overlap(out[i].p, out[i].bytes, x.p, x.bytes);
    for (int j = 0; j < i; ++j) shared |= overlap(out[i].p, out[i].bytes, out[j].p, out[j].bytes);
    if (shared) {
      set_error("uc_verify_draft: outputs overlap inputs or each other");
      return UC_ERR_ARG;
    }
  }
  VerifyParams p;
  memset(&p, 0, sizeof(p));
  p.target = target;
  p.draft = draft;
  p.target_b = target_b;
  p.target_t = target_t;
  p.draft_b = draft_b;
  p.draft_t = draft_t;
  p.tokens = tokens;
  p.n_draft = n_draft;
  p.u = u;
  p.noise = noise;
  p.accepted = accepted;
  p.out_tokens = out_tokens;
  p.logprob = logprob;
  p.batch = batch;
  p.n_tok = n_tok;
  p.vocab = vocab;
  p.greedy = greedy;
  const double inv = greedy ? 1.0 : 1.0 / temperature, scale = inv * 1.4426950408889634074;
  p.inv_temperature = (float)inv;
  p.scale = make_float2((float)scale, (float)(scale - (double)(float)scale));
  const int64_t rows = (int64_t)batch * (n_tok + 1 + (draft ? n_tok : 0)), vecs = row_vecs(vocab, element);
  const int64_t slots = kRowsPerSm * (int64_t)num_sms();
  // tiles of a row: the split that the SMs are through with first, a CTA's start and end as long as kStart vectors
  constexpr int64_t kStart = 2048;
  const int64_t most = std::min<int64_t>(kMostTiles, (vecs + kMinSpan - 1) / kMinSpan);
  int64_t least = INT64_MAX;
  for (int64_t t = 1; t <= most; ++t) {
    const int64_t span = (vecs + t - 1) / t, cost = (rows * t + slots - 1) / slots * (kStart + span);
    if (cost < least) {
      least = cost;
      p.span = (int)span;
    }
  }
  p.tiles = (int)((vecs + p.span - 1) / p.span);
  const int64_t pick = greedy ? 1 : std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(kPickMost, vocab / kPickMinSpan),
                                                                         kPickPerSm * (int64_t)num_sms() / batch));
  p.pick_span = (int)((vocab + pick - 1) / pick);
  p.pick_tiles = (int)((vocab + p.pick_span - 1) / p.pick_span);
  uint8_t* const w = static_cast<uint8_t*>(workspace);
  p.status = reinterpret_cast<DevStatus*>(w);
  p.best = reinterpret_cast<uint64_t*>(w + 256);
  p.part_ms = reinterpret_cast<float2*>(p.best + batch);
  p.part_at = reinterpret_cast<int32_t*>(p.part_ms + rows * p.tiles);
  p.done = p.part_at + rows * p.tiles;
  launch_verify(p, dtype, reinterpret_cast<cudaStream_t>(stream));
  return cuda_check(fn);
}

}  // extern "C"
