// What the kernels of attention with a window share: where a sequence's keys lie,
// and a row from its definition.
#pragma once

#include <climits>

#include "common.cuh"
#include "internal.h"

namespace uc {

constexpr float kLn2 = 0.69314718055994530942f;

// A sequence and its queries: query t has position first + t.
struct WindowSeq {
  int n, nq, first;
  int kept;  // positions from here on are in the cache, and the first ones
};

__device__ __forceinline__ WindowSeq window_seq(const WindowParams& p, int b) {
  const int n = p.lengths[b], nq = p.n_query ? p.n_query[b] : p.n_tok;
  WindowSeq s;
  s.n = max(n, 0);
  s.nq = min(max(nq, 0), p.n_tok);
  s.first = s.n - s.nq;
  s.kept = s.n > p.n_rows ? s.n - (p.n_rows - p.n_sink) : 0;
  return s;
}

// Reports counts out of range.
__device__ __forceinline__ void window_check(const WindowParams& p, int b) {
  const int nq = p.n_query ? p.n_query[b] : p.n_tok;
  if (p.lengths[b] < 0 || nq < 0 || nq > p.n_tok) set_status(p.status, UC_ERR_RANGE, b);
}

// The keys that queries at positions pa .. pb see between them: the first `sinks`
// tokens, then positions lo .. hi - 1. Of a sequence that has not filled its rows,
// lo is 0 where the window begins among the first tokens.
struct WindowKeys {
  int sinks, lo, hi;
  __device__ __forceinline__ int count() const { return sinks + hi - lo; }
  __device__ __forceinline__ int position(int i) const { return i < sinks ? i : lo + i - sinks; }
};

__device__ __forceinline__ WindowKeys window_keys(const WindowParams& p, const WindowSeq& s, int pa, int pb) {
  WindowKeys k;
  k.hi = max(pb + 1, 0);
  k.lo = max(max(pa - p.window + 1, 0), s.kept);
  k.sinks = p.n_sink;
  if (s.kept == 0 && k.lo <= p.n_sink) k.lo = k.sinks = 0;
  if (k.hi <= k.lo) {
    k.lo = k.hi;
    k.sinks = min(k.sinks, k.hi);
  }
  return k;
}

// The cache's row of a position that it holds.
__device__ __forceinline__ int window_row(const WindowParams& p, int pos) {
  if (pos < p.n_rows) return pos;
  return p.n_sink + (int)((uint32_t)(pos - p.n_sink) % (uint32_t)(p.n_rows - p.n_sink));
}

__device__ __forceinline__ bool window_sees(const WindowParams& p, int pos, int key) {
  return key <= pos && (pos - key < p.window || key < p.n_sink);
}

// The output of one query from its definition, key by key and with none that it
// does not see: for rows that a product over whole tiles left NaN or infinite (0 times what
// a masked row of v holds is not 0 there). A warp takes every `shares`-th run of four keys from
// `share` on; lane l has channels 4 l .. 4 l + 3. Sums relative to 2^m.
struct WindowPart {
  float4 o;
  float m, l;
};
static __device__ __noinline__ WindowPart window_row_part(const WindowParams& p, int b, int h, int t, int share,
                                                          int shares) {
  constexpr int kRun = 4;
  const int lane = threadIdx.x & 31, kvh = h / p.group;
  const WindowSeq s = window_seq(p, b);
  const int pos = s.first + t;
  const WindowKeys keys = window_keys(p, s, pos, pos);
  const int n = keys.count();
  const uint2 qw = *reinterpret_cast<const uint2*>(p.q.at(b, h, t) + 4 * lane);
  const float q[4] = {bf16_lo(qw.x), bf16_hi(qw.x), bf16_lo(qw.y), bf16_hi(qw.y)};
  float o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
  for (int64_t i = (int64_t)kRun * share; i < n; i += kRun * shares) {
    bool see[kRun];
    uint2 kw[kRun], vw[kRun];
    float x[kRun];
#pragma unroll
    for (int u = 0; u < kRun; ++u) {
      const int key = i + u < n ? keys.position((int)i + u) : INT_MAX;
      see[u] = window_sees(p, pos, key);
      kw[u] = vw[u] = make_uint2(0u, 0u);
      if (see[u]) {
        const int row = window_row(p, key);
        kw[u] = *reinterpret_cast<const uint2*>(p.k.at(b, kvh, row) + 4 * lane);
        vw[u] = *reinterpret_cast<const uint2*>(p.v.at(b, kvh, row) + 4 * lane);
      }
    }
#pragma unroll
    for (int u = 0; u < kRun; ++u)
      x[u] = q[0] * bf16_lo(kw[u].x) + q[1] * bf16_hi(kw[u].x) + q[2] * bf16_lo(kw[u].y) + q[3] * bf16_hi(kw[u].y);
#pragma unroll
    for (int d = 16; d; d >>= 1)
#pragma unroll
      for (int u = 0; u < kRun; ++u) x[u] += __shfl_xor_sync(0xffffffffu, x[u], d);
    float top = m;
#pragma unroll
    for (int u = 0; u < kRun; ++u) {
      x[u] = see[u] ? x[u] * p.scale_log2 : -INFINITY;
      top = fmaxf(top, x[u]);
    }
    const float base = top == -INFINITY ? 0.f : top, shrink = ex2_approx(m - base);
    l *= shrink;
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] *= shrink;
#pragma unroll
    for (int u = 0; u < kRun; ++u) {
      const float e = ex2_approx(x[u] - base);
      const float v[4] = {bf16_lo(vw[u].x), bf16_hi(vw[u].x), bf16_lo(vw[u].y), bf16_hi(vw[u].y)};
      l += e;
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] = fmaf(e, v[c], o[c]);
    }
    m = top;
  }
  return WindowPart{make_float4(o[0], o[1], o[2], o[3]), m, l};
}

struct WindowRow {
  float4 o;
  float lse;
};
__device__ __forceinline__ WindowRow window_row_of(const WindowPart& w) {
  const float inv = w.l == 0.f ? 0.f : 1.f / w.l;
  return WindowRow{make_float4(w.o.x * inv, w.o.y * inv, w.o.z * inv, w.o.w * inv),
                   w.l == 0.f ? -INFINITY : (w.m + log2f(w.l)) * kLn2};
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

// A finished row, by a warp: o (lane l: channels 4 l ..) and l relative to 2^m. An
// infinite l: neither is known.
__device__ __forceinline__ void window_store_row(const WindowParams& p, int b, int h, int t, float4 o, float m, float l) {
  const int lane = threadIdx.x & 31;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  float4 y = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  const bool bad = !(finite(y.x) && finite(y.y) && finite(y.z) && finite(y.w));
  float lse = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
  if (__any_sync(0xffffffffu, bad) && l == l) {
    const WindowRow w = window_row_of(window_row_part(p, b, h, t, 0, 1));
    y = w.o;
    if (!finite(l)) lse = w.lse;
  }
  *reinterpret_cast<uint2*>(p.out.at(b, h, t) + 4 * lane) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
  if (lane == 0 && p.lse != nullptr)
    p.lse[((int64_t)b * p.n_q_heads + h) * p.n_tok + t] = lse;
}

}  // namespace uc
