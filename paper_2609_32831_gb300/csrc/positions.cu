// Rotary positions of queries and keys, and new tokens into the cache of a
// layer with a sliding window.
//
// Pair i of a row at position p turns by p f_i: a' = s (a cos - b sin), b' = s (a
// sin + b cos). The angle is a fraction of a turn in 64 bits, p times f_i / 2 pi
// modulo one by integer arithmetic (2^-33 turns at the largest position), cut
// to an eighth of a turn around the nearest quarter before its sine and cosine
// are taken in fp32: as exact a million tokens into a context as at its start.
//
// Every row is read once and written once, so HBM bounds it. A thread holds the
// sines and cosines of its 16 bytes' pairs and walks the token's heads
// with them, four rows in flight; a token's heads go to several threads where
// tokens are few. 8 x 8192 tokens of 32 heads: 164 us, 97 % of the copy rate; 8 prompts
// of up to 4097 tokens into rings: 81 us, 92 % (their bytes take 75.0). Pairs (i, i + P) with P no multiple of
// a vector's elements take a warp per token, partners by shuffles: 244 us for 8 x 8192 tokens
// of 28 heads (their bytes: 139), a thread per pair of elements 295.
#include <climits>
#include <cmath>
#include <cstring>

#include "args.h"
#include "common.cuh"
#include "internal.h"

namespace uc {

namespace {

constexpr int kPosThreads = 128;

// Cosine and sine of p turns * 2^-64, times scale.
__device__ __forceinline__ float2 turned(int32_t p, uint64_t turn, float scale) {
  const uint64_t a = (uint64_t)(int64_t)p * turn;
  const uint32_t quarter = (uint32_t)((a + (1ull << 61)) >> 62);
  const int64_t rest = (int64_t)(a - ((uint64_t)quarter << 62));
  float s, c;
  sincospif((float)rest * 1.0842021724855044e-19f, &s, &c);  // 2^-63: in halves of a turn
  const float cc = quarter & 1 ? s : c, ss = quarter & 1 ? c : s;
  return make_float2((((quarter + 1) & 2) ? -cc : cc) * scale, ((quarter & 2) ? -ss : ss) * scale);
}

// 16 bytes of elements as fp32, and back.
template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int kE = 4;
  static __device__ __forceinline__ void get(const uint4& v, float* x) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 put(const float* x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
  static __device__ __forceinline__ float one(float x) { return x; }
  static __device__ __forceinline__ float back(float x) { return x; }
};
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int kE = 8;
  static __device__ __forceinline__ void get(const uint4& v, float* x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = bf16_lo(w[i]);
      x[2 * i + 1] = bf16_hi(w[i]);
    }
  }
  static __device__ __forceinline__ uint4 put(const float* x) {
    return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
  }
  static __device__ __forceinline__ float one(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __forceinline__ __nv_bfloat16 back(float x) { return __float2bfloat16_rn(x); }
};
template <>
struct Vec<__half> {
  static constexpr int kE = 8;
  static __device__ __forceinline__ void get(const uint4& v, float* x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ uint4 put(const float* x) {
    return make_uint4(pack_f16(x[0], x[1]), pack_f16(x[2], x[3]), pack_f16(x[4], x[5]), pack_f16(x[6], x[7]));
  }
  static __device__ __forceinline__ float one(__half x) { return __half2float(x); }
  static __device__ __forceinline__ __half back(float x) { return __float2half_rn(x); }
};

// Where a token's rows come from and go to.
struct Token {
  int b, t, pos;
  bool keep;  // its row of the cache is its own
  int slot;
};

__device__ __forceinline__ Token token_of(const PositionParams& p, int64_t i, bool first_thread) {
  Token k;
  k.b = (int)(i / p.n_tok);
  k.t = (int)(i - (int64_t)k.b * p.n_tok);
  k.keep = false;
  k.slot = 0;
  if (p.per_token) {
    k.pos = p.positions[i];
    return k;
  }
  const int first = p.positions[k.b];
  k.pos = (int)((uint32_t)first + (uint32_t)k.t);  // (wraps as int32 does; refused below where it is stored)
  if (p.out_total != nullptr) {
    const int n = p.n_new ? p.n_new[k.b] : p.n_tok;
    const bool ok = first >= 0 && n >= 0 && n <= p.n_tok && (int64_t)first + n <= INT32_MAX;
    if (k.t == 0 && first_thread) {
      if (!ok) set_status(p.status, UC_ERR_RANGE, k.b);
      p.out_total[k.b] = ok ? first + n : first;
    }
    k.keep = ok && k.t < n && (k.pos < p.n_sink || k.pos >= first + n - p.ring);
    k.slot = k.pos < p.n_sink ? k.pos : p.n_sink + (int)((uint32_t)(k.pos - p.n_sink) % (uint32_t)p.ring);
  }
  return k;
}

// fn(group, first head, heads) for the parts of the groups in heads [h0, h1).
template <typename F>
__device__ __forceinline__ void groups_in(const PositionParams& p, int h0, int h1, F&& fn) {
  int begin = 0;
#pragma unroll 1
  for (int g = 0; g < p.n_groups; ++g) {
    const int a = max(h0 - begin, 0), n = min(h1 - begin, p.g[g].heads) - a;
    if (n > 0) fn(p.g[g], a, n);
    begin += p.g[g].heads;
  }
}

// A thread: 2 vectors of a token's rows. INTER: vectors u and u + half the row.
// Else vectors u and u + P / kE where they are pairs, or two of the rest.
template <typename T, bool INTER>
__global__ void __launch_bounds__(kPosThreads) positions_kernel(const __grid_constant__ PositionParams p) {
  using V = Vec<T>;
  constexpr int kE = V::kE, kV = kHeadDim / kE, kUnits = kV / 2;
  constexpr int kRowsInFlight = 4;
  const int64_t tokens = (int64_t)p.batch * p.n_tok;
  const int64_t at = (int64_t)(blockIdx.x / p.parts) * (kPosThreads / kUnits) + threadIdx.x / kUnits;
  const int part = blockIdx.x % p.parts, u = threadIdx.x % kUnits;
  if (at >= tokens) return;
  const Token k = token_of(p, at, part == 0 && u == 0);
  const int h0 = (int)((int64_t)p.heads * part / p.parts), h1 = (int)((int64_t)p.heads * (part + 1) / p.parts);
  const int pv = INTER ? 0 : p.n_pairs / kE;           // vectors of first elements
  const bool pair = INTER || u < pv;
  const int va = INTER || u < pv ? u : u + pv, vb = INTER ? u + kUnits : u < pv ? u + pv : u + kUnits;
  // kE pairs: (element e of va, of vb), or elements (2 e, 2 e + 1) of va and then of vb
  float c[kE], s[kE];
  uint32_t live = 0;
  if (pair) {
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const int i = INTER ? (e < kE / 2 ? va * (kE / 2) + e : vb * (kE / 2) + e - kE / 2) : va * kE + e;
      if (i < p.n_pairs) {
        live |= 1u << e;
        const float2 cs = turned(k.pos, p.turn[i], p.scale);
        c[e] = cs.x;
        s[e] = cs.y;
      }
    }
  }
  auto turn = [&](uint4& wa, uint4& wb) {
    if (live == 0) return;
    float a[kE], b[kE];
    V::get(wa, a);
    V::get(wb, b);
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      float& x = INTER ? (e < kE / 2 ? a[2 * e] : b[2 * e - kE]) : a[e];
      float& y = INTER ? (e < kE / 2 ? a[2 * e + 1] : b[2 * e - kE + 1]) : b[e];
      const float x1 = fmaf(x, c[e], -y * s[e]), y1 = fmaf(x, s[e], y * c[e]);
      if (!INTER || (live >> e & 1)) {
        x = x1;
        y = y1;
      }
    }
    wa = V::put(a);
    wb = V::put(b);
  };
  groups_in(p, h0, h1, [&](const PositionGroup& g, int h, int n) {
    if (g.role != kTurn && !k.keep) return;
    const T* const src0 = reinterpret_cast<const T*>(g.src.base) + k.b * g.src.sb + k.t * g.src.st;
    T* const dst0 = reinterpret_cast<T*>(g.dst.base) + k.b * g.dst.sb + (g.role == kTurn ? k.t : k.slot) * g.dst.st;
    const bool turns = g.role != kStore;
#pragma unroll 1
    for (int i = h; i < h + n; i += kRowsInFlight) {
      uint4 a[kRowsInFlight], b[kRowsInFlight];
#pragma unroll
      for (int r = 0; r < kRowsInFlight; ++r)
        if (i + r < h + n) {
          const uint4* const row = reinterpret_cast<const uint4*>(src0 + (i + r) * g.src.sh);
          a[r] = row[va];
          b[r] = row[vb];
        }
#pragma unroll
      for (int r = 0; r < kRowsInFlight; ++r)
        if (i + r < h + n) {
          if (turns) turn(a[r], b[r]);
          uint4* const row = reinterpret_cast<uint4*>(dst0 + (i + r) * g.dst.sh);
          row[va] = a[r];
          row[vb] = b[r];
        }
    }
  });
}

// Four elements of a row: one lane's, as words.
template <typename T>
struct Four {
  static constexpr int kWords = 4 * sizeof(T) / 4;
  uint32_t w[kWords];
};

// Pairs (i, i + P) of any P: a warp per token, lane l has channels 4 l .. 4 l + 3.
// Their partners lie P channels on or back: in two lanes' words there, brought
// together and shifted by P mod 4 elements.
template <typename T>
__global__ void __launch_bounds__(kPosThreads) positions_any_kernel(const __grid_constant__ PositionParams p) {
  using V = Vec<T>;
  using F = Four<T>;
  constexpr int kPer = 4 / (int)sizeof(T);  // elements of a word
  const int64_t at = (int64_t)(blockIdx.x / p.parts) * (kPosThreads / 32) + threadIdx.x / 32;
  const int part = blockIdx.x % p.parts, lane = threadIdx.x & 31;
  if (at >= (int64_t)p.batch * p.n_tok) return;
  const Token k = token_of(p, at, part == 0 && lane == 0);
  const int h0 = (int)((int64_t)p.heads * part / p.parts), h1 = (int)((int64_t)p.heads * (part + 1) / p.parts);
  float c[4], s[4];
  bool first[4], live[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int ch = 4 * lane + e;
    first[e] = ch < p.n_pairs;
    live[e] = ch < 2 * p.n_pairs;
    const float2 cs = live[e] ? turned(k.pos, p.turn[first[e] ? ch : ch - p.n_pairs], p.scale) : make_float2(1.f, 0.f);
    c[e] = cs.x;
    s[e] = first[e] ? -cs.y : cs.y;
  }
  auto value = [](const F& f, int e) -> float {
    if constexpr (kPer == 1) {
      return __uint_as_float(f.w[e]);
    } else {
      const uint16_t x = (uint16_t)(f.w[e >> 1] >> (16 * (e & 1)));
      return V::one(*reinterpret_cast<const T*>(&x));
    }
  };
  // the four elements that begin `shift` channels behind a lane's first (any sign)
  auto moved = [&](const F& x, int shift) -> F {
    const int lanes = shift >> 2, rest = shift & 3;
    F a, b, r;
#pragma unroll
    for (int i = 0; i < F::kWords; ++i) {
      a.w[i] = __shfl_sync(0xffffffffu, x.w[i], (lane + lanes) & 31);
      b.w[i] = __shfl_sync(0xffffffffu, x.w[i], (lane + lanes + 1) & 31);
    }
    uint32_t w[2 * F::kWords];
#pragma unroll
    for (int i = 0; i < F::kWords; ++i) {
      w[i] = a.w[i];
      w[F::kWords + i] = b.w[i];
    }
    const int words = rest / kPer;
#pragma unroll
    for (int i = 0; i < F::kWords; ++i) {
      uint32_t lo = w[i], hi = w[i + 1];
#pragma unroll
      for (int y = 1; y < F::kWords; ++y)
        if (words == y) {
          lo = w[i + y];
          hi = i + y + 1 < 2 * F::kWords ? w[i + y + 1] : 0u;
        }
      r.w[i] = kPer == 2 && (rest & 1) ? __funnelshift_r(lo, hi, 16) : lo;
    }
    return r;
  };
  groups_in(p, h0, h1, [&](const PositionGroup& g, int h, int n) {
    if (g.role != kTurn && !k.keep) return;
    const T* const src0 = reinterpret_cast<const T*>(g.src.base) + k.b * g.src.sb + k.t * g.src.st + 4 * lane;
    T* const dst0 = reinterpret_cast<T*>(g.dst.base) + k.b * g.dst.sb + (g.role == kTurn ? k.t : k.slot) * g.dst.st + 4 * lane;
    constexpr int kRowsInFlight = 4;  // (eight took a tenth longer: what bounds it is instructions, 150 a row)
#pragma unroll 1
    for (int i = h; i < h + n; i += kRowsInFlight) {
      F x[kRowsInFlight];
#pragma unroll
      for (int r = 0; r < kRowsInFlight; ++r)
        if (i + r < h + n) {
          if constexpr (kPer == 1) {
            const uint4 w = *reinterpret_cast<const uint4*>(src0 + (i + r) * g.src.sh);
            x[r].w[0] = w.x; x[r].w[1] = w.y; x[r].w[2] = w.z; x[r].w[3] = w.w;
          } else {
            const uint2 w = *reinterpret_cast<const uint2*>(src0 + (i + r) * g.src.sh);
            x[r].w[0] = w.x; x[r].w[1] = w.y;
          }
        }
#pragma unroll
      for (int r = 0; r < kRowsInFlight; ++r)
        if (i + r < h + n) {
          if (g.role != kStore) {
            const F on = moved(x[r], p.n_pairs), back = moved(x[r], -p.n_pairs);
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              y[e] = fmaf(value(x[r], e), c[e], (first[e] ? value(on, e) : value(back, e)) * s[e]);
#pragma unroll
            for (int w = 0; w < F::kWords; ++w) {
              if constexpr (kPer == 1) {
                if (live[w]) x[r].w[w] = __float_as_uint(y[w]);
              } else {
                const T lo = V::back(y[2 * w]), hi = V::back(y[2 * w + 1]);
                uint32_t z = *reinterpret_cast<const uint16_t*>(&lo) | (uint32_t)*reinterpret_cast<const uint16_t*>(&hi) << 16;
                if (!live[2 * w]) z = (z & 0xffff0000u) | (x[r].w[w] & 0xffffu);
                if (!live[2 * w + 1]) z = (z & 0xffffu) | (x[r].w[w] & 0xffff0000u);
                x[r].w[w] = z;
              }
            }
          }
          if constexpr (kPer == 1)
            *reinterpret_cast<uint4*>(dst0 + (i + r) * g.dst.sh) = make_uint4(x[r].w[0], x[r].w[1], x[r].w[2], x[r].w[3]);
          else
            *reinterpret_cast<uint2*>(dst0 + (i + r) * g.dst.sh) = make_uint2(x[r].w[0], x[r].w[1]);
        }
    }
  });
}

template <typename T>
void launch_typed(PositionParams p, cudaStream_t st) {
  constexpr int kE = Vec<T>::kE;
  const bool vectors = p.interleaved || p.n_pairs % kE == 0;
  const int per = vectors ? kPosThreads / (kHeadDim / kE / 2) : kPosThreads / 32;
  const int64_t blocks = ((int64_t)p.batch * p.n_tok + per - 1) / per;
  // a token's heads to several threads, until the SMs are full
  const int64_t want = 8 * (int64_t)num_sms();
  p.parts = (int)std::min<int64_t>(p.heads, std::max<int64_t>(1, (want + blocks - 1) / blocks));
  const unsigned grid = (unsigned)(blocks * p.parts);
  if (!vectors)
    positions_any_kernel<T><<<grid, kPosThreads, 0, st>>>(p);
  else if (p.interleaved)
    positions_kernel<T, true><<<grid, kPosThreads, 0, st>>>(p);
  else
    positions_kernel<T, false><<<grid, kPosThreads, 0, st>>>(p);
  count_launch();
}

// freq / 2 pi modulo one, in 2^-64 turns. The product with 1 / 2 pi (given as two
// doubles) is formed as two doubles.
uint64_t turns_of(double freq) {
  constexpr double kHi = 0x1.45f306dc9c883p-3, kLo = -0x1.6b01ec5417056p-57;
  const double p = freq * kHi, rest = std::fma(freq, kHi, -p) + freq * kLo;
  // (both parts modulo one: [-1/2, 1/2), times 2^64 exactly; |p| < 2^29)
  auto part = [](double x) { return (uint64_t)std::llrint((x - (double)(int64_t)std::floor(x + 0.5)) * 0x1p64); };
  return part(p) + part(rest);
}

uc_status set_table(const uc_rotary_table* t, const char* fn, PositionParams* p) {
  if (t->n_pairs < 1 || t->n_pairs > UC_MAX_ROTARY_PAIRS || (t->interleaved != 0 && t->interleaved != 1) ||
      !std::isfinite(t->scale)) {
    set_error("%s: bad table (%d pairs, interleaved %d, scale %g)", fn, t->n_pairs, t->interleaved, t->scale);
    return UC_ERR_ARG;
  }
  for (int i = 0; i < t->n_pairs; ++i) {
    if (!(std::fabs(t->freq[i]) < 2147483648.0)) {
      set_error("%s: freq[%d] is not finite or too large", fn, i);
      return UC_ERR_ARG;
    }
    p->turn[i] = turns_of(t->freq[i]);
  }
  p->n_pairs = t->n_pairs;
  p->interleaved = t->interleaved;
  p->scale = (float)t->scale;
  return UC_OK;
}

bool same_rows(const RowsDev& a, const RowsDev& b) {
  return a.base == b.base && a.sb == b.sb && a.sh == b.sh && a.st == b.st;
}

// Tokens whose rows one launch can index.
bool fits(int batch, int n_tok, int heads) {
  return (int64_t)batch * n_tok <= (int64_t(1) << 32) / std::max(heads, 1);
}

}  // namespace

void launch_positions(const PositionParams& p, int dtype, cudaStream_t st) {
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

uc_status uc_rotary(const uc_rotary_table* table, const int32_t* positions, int32_t per_token, int32_t dtype,
                    int32_t batch, int32_t n_tok, const uc_rows* q, const uc_rows* q_out, int32_t n_q_heads,
                    const uc_rows* k, const uc_rows* k_out, int32_t n_kv_heads, void* stream) {
  UC_TRACE();
  const char* const fn = "uc_rotary";
  if (dtype != UC_FP32 && dtype != UC_BF16 && dtype != UC_FP16) {
    set_error("uc_rotary: bad type %d", dtype);
    return UC_ERR_ARG;
  }
  const bool both = k != nullptr;
  if (batch < 1 || n_tok < 1 || n_q_heads < 1 || n_q_heads > 65535 || (both && (n_kv_heads < 1 || n_kv_heads > 65535)) ||
      !fits(batch, n_tok, n_q_heads + (both ? n_kv_heads : 0))) {
    set_error("uc_rotary: unsupported shape (batch %d, tokens %d, heads %d and %d)", batch, n_tok, n_q_heads, n_kv_heads);
    return UC_ERR_SHAPE;
  }
  if (table == nullptr || positions == nullptr || !aligned(positions, 4) || both != (k_out != nullptr)) {
    set_error("uc_rotary: null or misaligned argument, or one of k and k_out");
    return UC_ERR_ARG;
  }
  PositionParams p;
  memset(&p, 0, sizeof(p));
  uc_status st = set_table(table, fn, &p);
  if (st != UC_OK) return st;
  const int element = dtype == UC_FP32 ? 4 : 2;
  const uc_rows* const in[2] = {q, k};
  const uc_rows* const out[2] = {q_out, k_out};
  const char* const names[2][2] = {{"q", "q_out"}, {"k", "k_out"}};
  uint64_t n_in[2], n_out[2];
  p.n_groups = both ? 2 : 1;
  for (int i = 0; i < p.n_groups; ++i) {
    PositionGroup& g = p.g[i];
    g.heads = i == 0 ? n_q_heads : n_kv_heads;
    g.role = kTurn;
    p.heads += g.heads;
    st = check_rows(in[i], fn, names[i][0], batch, g.heads, n_tok, &g.src, &n_in[i], element);
    if (st == UC_OK) st = check_rows(out[i], fn, names[i][1], batch, g.heads, n_tok, &g.dst, &n_out[i], element);
    if (st != UC_OK) return st;
  }
  const uint64_t n_pos = 4ull * batch * (per_token ? n_tok : 1);
  for (int i = 0; i < p.n_groups; ++i) {
    const RowSet o{&p.g[i].dst, {batch, p.g[i].heads, n_tok}, n_out[i], element};
    bool shared = rows_meet(o, o) || rows_meet(o, positions, n_pos);
    for (int j = 0; j < p.n_groups; ++j) {
      const RowSet x{&p.g[j].src, {batch, p.g[j].heads, n_tok}, n_in[j], element};
      shared |= !(i == j && same_rows(p.g[i].dst, p.g[i].src)) && rows_meet(o, x);
      if (j < i) {
        const RowSet y{&p.g[j].dst, {batch, p.g[j].heads, n_tok}, n_out[j], element};
        shared |= rows_meet(o, y);
      }
    }
    if (shared) {
      set_error("uc_rotary: %s overlaps inputs, another output or itself", names[i][1]);
      return UC_ERR_ARG;
    }
  }
  p.batch = batch;
  p.n_tok = n_tok;
  p.positions = positions;
  p.per_token = per_token != 0;
  launch_positions(p, dtype, reinterpret_cast<cudaStream_t>(stream));
  return cuda_check(fn);
}

uc_status uc_window_append(const uc_window_cache* cache, const uc_rows* k, const uc_rows* v, int32_t n_tok,
                           const int32_t* held, const int32_t* n_new, const uc_rotary_table* table,
                           const uc_rows* q, const uc_rows* q_out, int32_t n_q_heads, int32_t* out_total,
                           void* workspace, size_t workspace_bytes, void* stream) {
  UC_TRACE();
  const char* const fn = "uc_window_append";
  RowsDev ck, cv;
  uint64_t nck, ncv;
  uc_status st = check_window_cache(cache, fn, &ck, &cv, &nck, &ncv);
  if (st != UC_OK) return st;
  const uc_window_cache cut = within_rows(*cache);
  cache = &cut;
  const int batch = cache->batch, hkv = cache->n_kv_heads;
  if (n_tok < 1 || (q != nullptr && (n_q_heads < 1 || n_q_heads > 65535)) ||
      !fits(batch, n_tok, 2 * hkv + (q != nullptr ? n_q_heads : 0))) {
    set_error("uc_window_append: unsupported shape (%d tokens, %d query heads)", n_tok, n_q_heads);
    return UC_ERR_SHAPE;
  }
  if (held == nullptr || out_total == nullptr || !aligned(held, 4) || !aligned(n_new, 4) || !aligned(out_total, 4) ||
      (q != nullptr) != (q_out != nullptr) || (q != nullptr && table == nullptr)) {
    set_error("uc_window_append: null or misaligned argument, one of q and q_out, or q without a table");
    return UC_ERR_ARG;
  }
  st = check_workspace(workspace, workspace_bytes, 256, fn);
  if (st != UC_OK) return st;
  PositionParams p;
  memset(&p, 0, sizeof(p));
  if (table != nullptr) {
    st = set_table(table, fn, &p);
    if (st != UC_OK) return st;
  }
  // k, v and q in, where they go
  uint64_t n_in[3], n_out[3] = {nck, ncv, 0};
  int size[3] = {cache->n_rows, cache->n_rows, n_tok};
  const uc_rows* const in[3] = {k, v, q};
  const char* const names[3] = {"k", "v", "q"};
  p.n_groups = q != nullptr ? 3 : 2;
  for (int i = 0; i < p.n_groups; ++i) {
    PositionGroup& g = p.g[i];
    g.heads = i == 2 ? n_q_heads : hkv;
    g.role = i == 0 && table != nullptr ? kTurnStore : i == 2 ? kTurn : kStore;
    p.heads += g.heads;
    st = check_rows(in[i], fn, names[i], batch, g.heads, n_tok, &g.src, &n_in[i]);
    if (st == UC_OK && i == 2) st = check_rows(q_out, fn, "q_out", batch, g.heads, n_tok, &g.dst, &n_out[2]);
    if (st != UC_OK) return st;
  }
  p.g[0].dst = ck;
  p.g[1].dst = cv;
  bool shared = held == out_total;
  const struct { const void* p; uint64_t bytes; } counts[3] = {
      {held, 4ull * batch}, {n_new, n_new ? 4ull * batch : 0}, {out_total, 4ull * batch}};
  for (int i = 0; i < 2; ++i) shared |= overlap(counts[i].p, counts[i].bytes, out_total, 4ull * batch);
  for (int i = 0; i < p.n_groups; ++i) {
    const RowSet o{&p.g[i].dst, {batch, p.g[i].heads, size[i]}, n_out[i]};
    shared |= rows_meet(o, o);
    for (int j = 0; j < 3; ++j) shared |= counts[j].bytes && rows_meet(o, counts[j].p, counts[j].bytes);
    for (int j = 0; j < p.n_groups; ++j) {
      const RowSet x{&p.g[j].src, {batch, p.g[j].heads, n_tok}, n_in[j]};
      shared |= !(i == 2 && j == 2 && same_rows(p.g[2].dst, p.g[2].src)) && rows_meet(o, x);
      shared |= i == 0 && rows_meet(x, out_total, 4ull * batch);
      if (j < i) {
        const RowSet y{&p.g[j].dst, {batch, p.g[j].heads, size[j]}, n_out[j]};
        shared |= rows_meet(o, y);
      }
    }
  }
  if (shared) {
    set_error("uc_window_append: the cache, q_out or out_total overlaps inputs, another of them or itself");
    return UC_ERR_ARG;
  }
  p.batch = batch;
  p.n_tok = n_tok;
  p.positions = held;
  p.n_new = n_new;
  p.out_total = out_total;
  p.n_sink = cache->n_sink;
  p.ring = cache->n_rows - cache->n_sink;
  p.status = static_cast<DevStatus*>(workspace);
  launch_positions(p, UC_BF16, reinterpret_cast<cudaStream_t>(stream));
  return cuda_check(fn);
}

}  // extern "C"
