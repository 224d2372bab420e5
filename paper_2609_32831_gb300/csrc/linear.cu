// Linear attention with a decay for each KV head over a state of constant
// size: per sequence and KV head, with gamma = exp(log_decay) <= 1,
//   S_t = gamma S_{t-1} + k_t v_t^T        (128 x 128, fp32)
//   o_t = S_t^T q_t / sqrt(128)            for every query head of the KV head.
#include <mutex>

#include "common.cuh"
#include "internal.h"
#include "tcgen05.cuh"

namespace uc {

// ------------------------------------------------------ token by token
// One CTA per (sequence, KV head, 32 value channels): a state column needs
// its own value channel only, so column slices are independent. Warp w holds
// rows (key channels) 16 w .. 16 w + 15, lane l the column 32 slice + l; the
// partial sums over a warp's rows meet in shared memory. Everything is loaded
// before the first token is taken: the state into registers, k, v and (where
// they fit) q of all tokens into shared memory. Bound by HBM in large batches:
// 64 sequences of 4 heads, 34.6 MB: 8.1 us, 4.3 TB/s; by the latency of its
// loads and one reduction per token in small ones (one sequence: 3.3 us).
// (Loads token by token: 0.6 and 0.4 us more, five tokens of 8 x 16 heads 2 us
// more than their 7.5.)
constexpr int kStepCols = 32;
constexpr int kStepWarps = 8;
constexpr int kStepRows = kHeadDim / kStepWarps;
constexpr int kStepHeads = 8;   // query heads reduced at a time
constexpr int kStepQRows = 64;  // rows of q in shared memory

__global__ void __launch_bounds__(32 * kStepWarps) linear_step_kernel(const __grid_constant__ LinearParams p) {
  __shared__ __align__(16) __nv_bfloat16 qs[kStepQRows][kHeadDim];
  __shared__ __align__(16) __nv_bfloat16 ks[UC_MAX_QTOKENS][kHeadDim];
  __shared__ __nv_bfloat16 vs[UC_MAX_QTOKENS][kStepCols];
  __shared__ float part[2][kStepHeads][kStepWarps][kStepCols];  // in turns
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr int kSlices = kHeadDim / kStepCols;
  const int bh = blockIdx.x / kSlices, slice = blockIdx.x % kSlices;
  const int b = bh / p.n_kv_heads, kvh = bh % p.n_kv_heads;
  const int n = min(p.lengths[b], p.n_tok);
  // gamma as two fp32 parts: rounded to one, a decay that remembers thousands
  // of tokens would drift by their number times 2^-25
  const float g_hi = p.decay[kvh].x, g_lo = p.decay[kvh].y;
  float s[kStepRows];
  const size_t at = ((size_t)bh * kHeadDim + warp * kStepRows) * kHeadDim + slice * kStepCols + lane;
#pragma unroll
  for (int r = 0; r < kStepRows; ++r) s[r] = p.state_in ? p.state_in[at + (size_t)r * kHeadDim] : 0.f;
  constexpr int kRow16 = kHeadDim / 8;  // 16-byte pieces of a row
  for (int i = tid; i < n * kRow16; i += 32 * kStepWarps)
    reinterpret_cast<uint4*>(ks[i / kRow16])[i % kRow16] =
        reinterpret_cast<const uint4*>(p.k.at(b, kvh, i / kRow16))[i % kRow16];
  for (int i = tid; i < n * kStepCols; i += 32 * kStepWarps)
    vs[i / kStepCols][i % kStepCols] = p.v.at(b, kvh, i / kStepCols)[slice * kStepCols + i % kStepCols];
  auto load_q = [&](int rows, auto&& from) {  // rows of q, the t and head of each by from()
    for (int i = tid; i < rows * kRow16; i += 32 * kStepWarps) {
      const int2 th = from(i / kRow16);
      reinterpret_cast<uint4*>(qs[i / kRow16])[i % kRow16] =
          reinterpret_cast<const uint4*>(p.q.at(b, kvh * p.group + th.y, th.x))[i % kRow16];
    }
  };
  const bool all = p.n_tok * p.group <= kStepQRows;
  if (all) load_q(n * p.group, [&](int i) { return make_int2(i / p.group, i % p.group); });
  __syncthreads();
  int turn = 0;
  for (int t = 0; t < p.n_tok; ++t) {
    if (t < n) {
      const float v = __bfloat162float(vs[t][lane]);
#pragma unroll
      for (int r = 0; r < kStepRows; r += 8) {
        const uint4 k8 = *reinterpret_cast<const uint4*>(&ks[t][warp * kStepRows + r]);
        const uint32_t w[4] = {k8.x, k8.y, k8.z, k8.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          s[r + 2 * u] = fmaf(s[r + 2 * u], g_hi, fmaf(s[r + 2 * u], g_lo, bf16_lo(w[u]) * v));
          s[r + 2 * u + 1] = fmaf(s[r + 2 * u + 1], g_hi, fmaf(s[r + 2 * u + 1], g_lo, bf16_hi(w[u]) * v));
        }
      }
    }
    for (int h0 = 0; h0 < p.group; h0 += kStepHeads, turn ^= 1) {
      const int nh = min(kStepHeads, p.group - h0);
      if (!all && t < n) {
        __syncthreads();  // (the last heads' q has been read)
        load_q(nh, [&](int i) { return make_int2(t, h0 + i); });
        __syncthreads();
      }
      if (t < n) {
        const int row = all ? t * p.group + h0 : 0;
        for (int h = 0; h < nh; ++h) {
          float o = 0.f;
#pragma unroll
          for (int r = 0; r < kStepRows; r += 8) {
            const uint4 q8 = *reinterpret_cast<const uint4*>(&qs[row + h][warp * kStepRows + r]);
            const uint32_t w[4] = {q8.x, q8.y, q8.z, q8.w};
#pragma unroll
            for (int u = 0; u < 4; ++u) o = fmaf(bf16_hi(w[u]), s[r + 2 * u + 1], fmaf(bf16_lo(w[u]), s[r + 2 * u], o));
          }
          part[turn][h][warp][lane] = o;
        }
      }
      __syncthreads();
      for (int i = tid; i < nh * kStepCols; i += 32 * kStepWarps) {
        float o = 0.f;
        if (t < n)
#pragma unroll
          for (int w = 0; w < kStepWarps; ++w) o += part[turn][i / kStepCols][w][i % kStepCols];
        // a token behind the sequence's end has no output: zero
        p.out.at(b, kvh * p.group + h0 + i / kStepCols, t)[slice * kStepCols + i % kStepCols] =
            __float2bfloat16_rn(o * p.scale);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < kStepRows; ++r) p.state_out[at + (size_t)r * kHeadDim] = s[r];
}

void launch_linear_step(const LinearParams& p, cudaStream_t st) {
  linear_step_kernel<<<p.batch * p.n_kv_heads * (kHeadDim / kStepCols), 32 * kStepWarps, 0, st>>>(p);
  count_launch();
}

// ----------------------------------------------------------------- chunks
// Prompts. With S the state before a chunk of kChunk tokens, i, j positions in
// it and nv its valid tokens,
//   o_i  = a_i (q_i S + sum_{j <= i} (q_i . k_j) gamma^{-(j+1)} v_j) / sqrt(128),  a_i = gamma^{i+1}
//   S'   = gamma^nv S + sum_j k_j (gamma^{nv-1-j} v_j)^T
// so a chunk costs Q K^T, Q S and P V per query head, the last two into one
// accumulator and with S and P in two parts (five 128^3 products), and one with
// three parts per KV head for the state. The floor is HBM: 64 KB of q and o per
// head and chunk, 1.5 us of an SM's share, against 5 x 512 cycles of the tensor
// pipe. What bounds it are a tile's products and the hand-overs between warps, one
// after the other: with seven heads o read, Q S, P V (4300 to 4900 cycles a tile),
// with one head those of the state's update (11.6 thousand cycles a chunk).
// 8 x 8192 tokens, 28 query and 4 KV heads: 330 us, 3.3 TB/s of q, k, v and o;
// 16 x up to 4097 tokens of 16 heads: 229 us, 2.8 TB/s; 131072 tokens: 591 us,
// 3.6 TB/s.
//
// One CTA per (sequence, KV head, run of chunks, part of its query heads):
//   WG0, WG1 (warps 0-7) halves of the columns of Q K^T: P = mask and weights,
//            two bf16 parts, back to tensor memory
//   WG2, WG3 (8-15) the epilogue, halves of the channels: o scaled, rounded and
//            stored, turned around in shared memory so that two lanes write a
//            32-byte sector of a row
//   WG4      (16-19) the state. It stays in tensor memory in fp32; per chunk
//            its bf16 copy goes to shared memory for Q S, and in bf16 what that
//            rounding left; in fp32 that stays behind, scaled by gamma^nv, and the
//            chunk's decayed values are formed in slices of 16 tokens (with one or
//            two heads the odd ones by WG0 and WG1) that accumulate on the rest
//            while the chunk's tiles run; the copy joins them, scaled, in fp32.
//            (The tensor cores' sums are cut, not rounded: 24 of them per chunk on
//            the whole state pulled it towards zero by up to 1.2e-5 of its size
//            where gamma is near 1; on the rest they cost 1e-7 of the chunk's own
//            sum.)
//   warp 20  TMA producer: k and v tiles per chunk and a q tile per head, in the
//            order they are needed, each into whichever slot is free
//   warp 21  issues Q K^T, one tile ahead
//   warp 22  issues Q S and P V (a chunk's first tile: P V and Q S)
//   warp 23  issues the slices' products and releases the chunk's k and v slots
//            (one warp for all of it: its own waits and issues took 3500 cycles a tile)
// In a sequence's last chunk, warps 21 and 22 first zero the k and v rows behind
// its end: they may hold NaN, and 0 x NaN is not 0. For the same reason a NaN or
// infinity in v would reach earlier tokens through P V, where their P is 0. So
// WG0 and WG1 look a chunk's v through beside its first P (on the issuing warp,
// between two products, 7 % of 8 x 8192 tokens). Where they find any, the
// chunk's slices are formed first (the state takes them as they are), warp 22
// puts zeros in their place before P V, and behind its last tile the CTA makes NaN
// of a channel's outputs from the token on that held one (1 % in all; code for it
// in the epilogue's loop: 5 to 14 %).
// Order of the products: Q K^T of the next tile while the epilogue reads the
// last one's o, then Q S and P V. (With the epilogue and the update on the
// warps that form P, and rows stored from registers, 32 lines per instruction,
// a tile took a third longer and an update of the state 6500 cycles.)
//
// Roundings to bf16: the output's own, 1.66e-3 of its norm, is the only one that
// shows. P and the copy of S that Q multiplies enter as two bf16 parts each (16
// bits); with one part each the output's error was 2.34e-3, with P alone in two
// 2.18e-3. That took 266 us instead of 330 for 8 x 8192 tokens and 208 instead of 229
// for 16 x up to 4097: two products fewer per tile, and 32 KB for a fifth slot (20 of
// the 64 us). None on the state's path: the decayed values enter as three bf16 parts
// (all 24 bits of v gamma^n; two parts left the state 2.7e-6 off), the update
// accumulates in fp32.
//
// a_i and gamma^{-(j+1)} take the row's common factor out of both products.
// Where gamma^128 < 2^-64 (a memory of under two tokens) a_i stops at 2^-64 and
// P carries gamma^{i-j} / a_i instead; Q S is then kept 2^-64 of its size where
// it should be less still.
constexpr int kLThreads = 768;
constexpr int kLRegLaunch = 80;  // registers per thread at launch, and after the warpgroups rebalance
constexpr int kLRegP = 88;
constexpr int kLRegEpilogue = 72;
constexpr int kLRegState = 80;
constexpr int kLRegOther = 72;
static_assert(256 * (kLRegP + kLRegEpilogue) + 128 * (kLRegState + kLRegOther) <= kLThreads * kLRegLaunch, "register split");
constexpr int kWarpEpilogue = 8, kWarpState = 16, kWarpTma = 20, kWarpQk = 21, kWarpMma = 22, kWarpSlice = 23;
constexpr uint32_t kTmemLinear = 512;
constexpr uint32_t kColOut = 256;    // o; the S slots are columns 0 and 128
constexpr uint32_t kColState = 384;
constexpr uint32_t kTileBytes = kChunk * kHeadDim * 2;
constexpr int kSlice = 16;  // tokens of one slice of decayed values
constexpr int kSlices = kChunk / kSlice;
constexpr uint32_t kSliceBytes = kSlice * kHeadDim * 2;
constexpr float kLeastScale = 5.421010862427522e-20f;  // 2^-64
constexpr int kHelpHeads = 2;  // query heads up to which WG0 and WG1 form the odd slices
constexpr int kLSlots = 4;
constexpr int kLFull = 8;  // "arrived" barriers, by load number: more than loads in flight

template <int N>
__device__ __forceinline__ void rebalance() {
  if constexpr (N < kLRegLaunch) setmaxnreg_dec<N>();
  if constexpr (N > kLRegLaunch) setmaxnreg_inc<N>();
}

struct LinearSmem {
  uint8_t slot[kLSlots][kTileBytes];   // [2 x 64 channels][128 tokens][128 B], 128B swizzle
  uint8_t s_rest[kTileBytes];          // what s leaves of it, the same
  uint8_t s[kTileBytes];               // the chunk's state, bf16 [2 x 64 value channels][128 key channels][128 B]
  uint8_t part[2][3][kSliceBytes];     // decayed values, three parts: [2 x 64 channels][16 tokens][128 B]
  uint4 turn[8][32 * 2];               // per epilogue warp: 32 rows of 32 B
  float pw[kChunk + 4];                // gamma^n
  float cj[kChunk];                    // gamma^{-(n + 1)}
  uint64_t full[kLFull], empty[kLSlots];
  uint64_t s_full[2], p_full[2], o_full[2], o_free;
  uint64_t st_ready, s_free, chunk_go[2], k_done[2], v_done[2], kv_done, part_full[2], part_free[2];
  uint32_t tmem_base;
  uint32_t ks[2], vs[2];               // slots of a chunk's k and v, by parity
  uint64_t drain[3];                   // the issuing warps' last products
  uint64_t v_hit[2];                   // a byte per warp that found NaN or infinities in its part of the chunk's v
  uint32_t v_odd;                      // some did, in any chunk
  int loads;                           // loads issued
  DevStatus status;                    // of this CTA's waits
  uint8_t slot_of[16];                 // slot of load L at L mod 16
};
static_assert(sizeof(LinearSmem) + 1024 <= 232448, "linear attention shared memory");

// gamma^n to fp32 rounding (n < 0 only where it stays finite): the exponent n log2(gamma) is formed from
// two fp32 parts of log2(gamma) and split into its whole part and a rest of at
// most 1/2 (in one fp32 number its error grows with n). n = 0 gives 1, also
// where gamma is 0.
__device__ __forceinline__ float decay_pow(float2 log2_gamma, int n) {
  const float m = (float)n;
  const float x = log2_gamma.x * m;
  if (x < -160.f) return 0.f;  // below the smallest fp32 subnormal
  const float w = rintf(x);
  const float rest = (x - w) + fmaf(log2_gamma.y, m, fmaf(log2_gamma.x, m, -x));
  return ldexpf(exp2f(rest), (int)w);
}

// One arrival for a warp whose lanes have all done their part: 32 arrivals of
// one instruction are taken one after the other.
__device__ __forceinline__ void warp_arrive(uint64_t* bar, int lane) {
  __syncwarp();
  if (lane == 0) mbar_arrive(bar);
}

__device__ __forceinline__ void tma_load_rows(void* dst, const CUtensorMap* map, int c0, int t, int h, int b,
                                              uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(t), "r"(h), "r"(b), "r"(smem_u32(bar))
      : "memory");
}

// A tile of kChunk rows from token t on: two loads of 64 channels.
__device__ __forceinline__ void load_tile(uint8_t* dst, const CUtensorMap* map, int t, int h, int b, uint64_t* bar) {
  mbar_arrive_expect_tx(bar, kTileBytes);
  tma_load_rows(dst, map, 0, t, h, b, bar);
  tma_load_rows(dst + kTileBytes / 2, map, 64, t, h, b, bar);
}

// One K = 16 step: D (+)= A B, descriptors as the low words of their bases.
__device__ __forceinline__ void issue_ss(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t id,
                                         uint32_t acc) {
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      ".reg .b64 da, db;\n"
      "setp.ne.b32 q, %6, 0;\n"
      "setp.ne.b32 p, %5, 0;\n"
      "mov.b64 da, {%1, %3};\n"
      "mov.b64 db, {%2, %3};\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n"
      "}\n" ::"r"(d),
      "r"(a), "r"(b), "r"(hi), "r"(id), "r"(acc), "r"(lead)
      : "memory");
}
__device__ __forceinline__ void issue_ts(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t id,
                                         uint32_t acc) {
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      ".reg .b64 db;\n"
      "setp.ne.b32 q, %5, 0;\n"
      "setp.ne.b32 p, %6, 0;\n"
      "mov.b64 db, {%2, %3};\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n"
      "}\n" ::"r"(d),
      "r"(a), "r"(b), "r"(hi), "r"(id), "r"(lead), "r"(acc)
      : "memory");
}
// The three products of a tile, in loops of one step each: 24 warps share the
// instruction caches, and straight-line issues were fetched anew every time.
// S = Q K^T: both along their 128-B rows (32 B per step, then the second 64 channels).
__device__ __forceinline__ void issue_q_k(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t id) {
#pragma unroll 1
  for (uint32_t k = 0; k < 8; ++k) {
    const uint32_t off = (k & 3) * 2 + (k >> 2) * (kTileBytes >> 5);
    issue_ss(lead, d, a + off, b + off, hi, id, k);
  }
}
// O (+)= Q S: the state's key channels along its rows (16 rows of 128 B per step).
__device__ __forceinline__ void issue_q_s(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t id,
                                          uint32_t acc) {
#pragma unroll 1
  for (uint32_t k = 0; k < 8; ++k)
    issue_ss(lead, d, a + (k & 3) * 2 + (k >> 2) * (kTileBytes >> 5), b + 128 * k, hi, id, acc | k);
}
// O (+)= P V: the two parts of P of 16 keys, eight columns each, lie where their S
// was read from.
__device__ __forceinline__ void issue_p_v(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t id,
                                          uint32_t acc) {
#pragma unroll 1
  for (uint32_t k = 0; k < 16; ++k) issue_ts(lead, d, a + 8 * k, b + 128 * (k >> 1), hi, id, acc | k);
}

// The decayed values of tokens ROWS sl .. ROWS sl + ROWS - 1 of a chunk as
// three bf16 parts ([2 x 64 channels][ROWS][128 B] each), by THREADS threads.
// Token j's weight w(j), 0 from nv on (whatever the row holds).
template <int ROWS, int THREADS, typename W>
__device__ __forceinline__ void decay_slice(const uint8_t* v, uint8_t (*parts)[ROWS * kHeadDim * 2], int sl, int nv,
                                            int thread, const W& weight) {
#pragma unroll 2
  for (int i = thread; i < 2 * ROWS * 8; i += THREADS) {
    const int half = i / (8 * ROWS), in = i % (8 * ROWS), j = ROWS * sl + (in >> 3);
    uint32_t part[3][4] = {};
    if (j < nv) {
      const float w = weight(j);
      const uint4 x = *(reinterpret_cast<const uint4*>(v + half * (kTileBytes / 2) + ROWS * sl * 128) + in);
      const uint32_t bits[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        // eight bits of the fp32 value per part, by cutting: nothing is left
        float a = bf16_lo(bits[e]) * w, b = bf16_hi(bits[e]) * w;
#pragma unroll
        for (int u = 0; u < 3; ++u) {
          const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
          part[u][e] = __byte_perm(x, y, 0x7632);
          a -= __uint_as_float(x & 0xffff0000u);
          b -= __uint_as_float(y & 0xffff0000u);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < 3; ++u)
      reinterpret_cast<uint4*>(parts[u])[i] = make_uint4(part[u][0], part[u][1], part[u][2], part[u][3]);
  }
  __syncwarp();
}

// D += K^T V over one slice: A the slice's rows of k, B its three parts.
__device__ __forceinline__ void issue_slice(uint32_t lead, uint32_t d, uint32_t k, uint32_t parts, uint32_t hi, uint32_t id) {
#pragma unroll 1
  for (uint32_t u = 0; u < 3; ++u) issue_ss(lead, d, k, parts + u * (kSliceBytes >> 4), hi, id, 1u);
}

// Two values as bf16 and as bf16 of what that leaves.
__device__ __forceinline__ void two_parts(float a, float b, uint32_t& whole, uint32_t& rest) {
  whole = pack_bf16(a, b);
  f2_unpack(f2_fma(f2_pack(bf16_lo(whole), bf16_hi(whole)), f2_pack(-1.f, -1.f), f2_pack(a, b)), a, b);
  rest = pack_bf16(a, b);
}

// Zeroes rows nv .. 127 of a tile, by one warp.
__device__ __forceinline__ void zero_rows(uint8_t* tile, int nv, int lane) {
  for (int half = 0; half < 2; ++half)
    for (int i = nv * 8 + lane; i < kChunk * 8; i += 32)
      reinterpret_cast<uint4*>(tile + half * (kTileBytes / 2))[i] = make_uint4(0, 0, 0, 0);
  fence_proxy_async_smem();
  __syncwarp();
}

// Do rows 0 .. nv - 1 of a tile hold NaN or infinities? 0 times them is NaN, and
// so is what it is added to. A warp's share of eight, by all of its lanes.
__device__ __forceinline__ bool holds_not_finite(const uint8_t* tile, int nv, int thread) {
  const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
  __nv_bfloat162 sum[4] = {zero, zero, zero, zero};
#pragma unroll
  for (int k = 0; k < (int)(kTileBytes / 16 / 256); ++k) {
    const int i = 256 * k + thread;  // 16 bytes: half, row, piece of the row's half
    uint4 x = make_uint4(0, 0, 0, 0);
    if ((i >> 3) % kChunk < nv) x = reinterpret_cast<const uint4*>(tile)[i];
    sum[0] = __hfma2(reinterpret_cast<__nv_bfloat162&>(x.x), zero, sum[0]);
    sum[1] = __hfma2(reinterpret_cast<__nv_bfloat162&>(x.y), zero, sum[1]);
    sum[2] = __hfma2(reinterpret_cast<__nv_bfloat162&>(x.z), zero, sum[2]);
    sum[3] = __hfma2(reinterpret_cast<__nv_bfloat162&>(x.w), zero, sum[3]);
  }
  const __nv_bfloat162 all = __hadd2(__hadd2(sum[0], sum[1]), __hadd2(sum[2], sum[3]));
  return __any_sync(0xffffffffu, __hisnan(all.x) || __hisnan(all.y));
}

// The elements of eight that are NaN or infinite, as a mask.
__device__ __forceinline__ uint32_t not_finite(const uint4& x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t mask = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) mask |= (uint32_t)((~(w[e >> 1] >> (16 * (e & 1))) & 0x7f80u) == 0u) << e;
  return mask;
}

// Zeroes those of a tile, by one warp.
__device__ __forceinline__ void clear_not_finite(uint8_t* tile, int lane) {
#pragma unroll 1
  for (int i = lane; i < (int)(kTileBytes / 16); i += 32)
    if (const uint32_t odd = not_finite(reinterpret_cast<const uint4*>(tile)[i]))
      for (int e = 0; e < 8; ++e)
        if ((odd >> e) & 1u) reinterpret_cast<uint16_t*>(tile)[8 * i + e] = 0;
  fence_proxy_async_smem();
  __syncwarp();
}

// The sequence of run `grun`.
__device__ __forceinline__ int sequence_of(const LinearPlan& plan, int batch, int grun) {
  int lo = 0, hi = batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (plan.run_begin[mid] <= grun) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Where a wait ran out in any warp, the others may have left their loops with copies
// and products still in flight: neither shared nor tensor memory is given back
// under them. By all threads behind a barrier (a role's lanes are apart before
// it), with the ordinary limit (the call's may be too short for it). The CTA's
// waits record in shared memory, so that its end knows of them without a register
// in any role; they reach the call's status word here.
__device__ __forceinline__ void drain_cta(LinearSmem& sm, DevStatus* status, int withhold, int warp) {
  if (threadIdx.x == 0) set_status(status, sm.status.code, sm.status.detail);
  bool gone = false;
  if (warp == kWarpTma) {
    const int loads = sm.loads;
#pragma unroll 1
    for (int i = max(0, loads - kLSlots); i < loads; ++i)
      if (i != withhold) dwait_warp(&sm.full[i % kLFull], (i / kLFull) & 1, status, 52, gone);
  } else if (warp > kWarpTma) {
    uint64_t* const bar = &sm.drain[warp - kWarpQk];
    umma_commit_lead(elect_one(), bar);  // (behind what its elected lane has issued)
    dwait_warp(bar, 0, status, 53, gone);
  }
  __syncthreads();
}

// What a CTA takes: a run of chunks of a KV head, and a part of its query heads.
struct LinearTask {
  int b, kvh, grun, h0, nh, len, c0, chunks, part;
};
__device__ __forceinline__ LinearTask linear_task(const LinearChunkParams& c, int cta) {
  const LinearParams& p = c.p;
  LinearTask k;
  k.part = cta % c.plan.head_parts;
  k.kvh = cta / c.plan.head_parts % p.n_kv_heads;
  k.grun = cta / (c.plan.head_parts * p.n_kv_heads);
  k.b = sequence_of(c.plan, p.batch, k.grun);
  k.h0 = k.part * c.plan.heads_per_part;
  k.nh = min(c.plan.heads_per_part, p.group - k.h0);
  k.len = p.lengths[k.b];
  k.c0 = (k.grun - c.plan.run_begin[k.b]) * c.plan.chunks_per_run;
  k.chunks = min(c.plan.chunks_per_run, (k.len + kChunk - 1) / kChunk - k.c0);  // chunks with a valid token
  return k;
}

// Makes NaN of a CTA's outputs in the channels, and from the token on, where v is
// not finite (what comes behind its run has it from the state). `first` is shared.
// The CTA's task is worked out anew: nothing has to be kept for it. Rolled loops:
// warps call it with the registers that their role left them, 72 at least (as a
// kernel it takes 25).
__device__ __noinline__ void spoil_outputs(const LinearChunkParams& c, int cta, int* first) {
  const LinearParams& p = c.p;
  const LinearTask k = linear_task(c, cta);
  const int t0 = k.c0 * kChunk, t1 = min(k.len, (k.c0 + k.chunks) * kChunk);
  if (threadIdx.x < kHeadDim) first[threadIdx.x] = t1;
  __syncthreads();
  constexpr int kPieces = kHeadDim / 8;
  const int piece = threadIdx.x % kPieces;
#pragma unroll 1
  for (int t = t0 + threadIdx.x / kPieces; t < t1; t += kLThreads / kPieces) {
    const uint32_t odd = not_finite(reinterpret_cast<const uint4*>(p.v.at(k.b, k.kvh, t))[piece]);
#pragma unroll 1
    for (int e = 0; e < 8; ++e)
      if ((odd >> e) & 1u) atomicMin(first + 8 * piece + e, t);
  }
  __syncthreads();
#pragma unroll 1
  for (int t = t0 + threadIdx.x / kPieces; t < t1; t += kLThreads / kPieces)
#pragma unroll 1
    for (int e = 0; e < 8; ++e)
      if (t >= first[8 * piece + e])
#pragma unroll 1
        for (int h = 0; h < k.nh; ++h)
          p.out.at(k.b, k.kvh * p.group + k.h0 + h, t)[8 * piece + e] = __ushort_as_bfloat16(0x7fff);
}

__global__ void __launch_bounds__(kLThreads, 1) linear_chunk_kernel(const __grid_constant__ LinearChunkParams c) {
  extern __shared__ uint8_t dyn_smem[];
  LinearSmem& sm = *reinterpret_cast<LinearSmem*>(
      (reinterpret_cast<uintptr_t>(dyn_smem) + 1023) & ~static_cast<uintptr_t>(1023));
  const LinearParams& p = c.p;
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const LinearTask task = linear_task(c, blockIdx.x);
  const int part = task.part, kvh = task.kvh, grun = task.grun, b = task.b, h0 = task.h0, nh = task.nh, len = task.len;
  const int c0 = task.c0, nc = task.chunks;
  const int tiles = nc * nh;
  // with few heads the update's chain of steps is longer than the tiles': WG0 and
  // WG1 take a part of it (one head, 16 x up to 4097 tokens: 239 -> 233 us when it was added; with
  // seven heads their tiles would wait for it: 267 -> 289 us for 8 x 8192)
  const bool help = nh <= kHelpHeads;
  // a sequence's last run ends with the state behind its last token
  const bool last_state = part == 0 && grun + 1 == c.plan.run_begin[b + 1];
  auto valid = [&](int ci) { return min(kChunk, len - (c0 + ci) * kChunk); };
  // loads in order, nh + 2 per chunk: k, the first head's q, v, the other heads' q
  auto load_k = [&](int ci) { return ci * (nh + 2); };
  auto load_v = [&](int ci) { return ci * (nh + 2) + 2; };
  auto load_q = [&](int ci, int h) { return ci * (nh + 2) + (h == 0 ? 1 : h + 2); };
  if (threadIdx.x == 0) {
    for (int s = 0; s < kLFull; ++s) mbar_init(&sm.full[s], 1);
    for (int s = 0; s < kLSlots; ++s) mbar_init(&sm.empty[s], 1);
    for (int s = 0; s < 2; ++s) {
      mbar_init(&sm.s_full[s], 1);
      mbar_init(&sm.o_full[s], 1);
      mbar_init(&sm.p_full[s], 8);     // (arrivals: one per warp)
      mbar_init(&sm.part_full[s], help && s == 1 ? 8 : 4);
      mbar_init(&sm.part_free[s], 1);
      mbar_init(&sm.chunk_go[s], 1);
      mbar_init(&sm.k_done[s], 1);
      mbar_init(&sm.v_done[s], 1);
    }
    mbar_init(&sm.o_free, 8);
    mbar_init(&sm.st_ready, 4);
    mbar_init(&sm.s_free, 1);
    mbar_init(&sm.kv_done, 1);
    for (int s = 0; s < 3; ++s) mbar_init(&sm.drain[s], 1);
    fence_barrier_init();
    sm.v_odd = 0;
    sm.loads = 0;
    sm.status.code = 0;
  }
  const float2 l2 = p.log2_decay[kvh];
  const bool strong = l2.x * kChunk < -64.f;
  if (threadIdx.x <= kChunk) {
    const float w = decay_pow(l2, threadIdx.x);
    sm.pw[threadIdx.x] = w;
    if (threadIdx.x < kChunk) sm.cj[threadIdx.x] = strong ? 0.f : decay_pow(l2, -1 - (int)threadIdx.x);
  }
  if (warp == kWarpMma) tmem_alloc(&sm.tmem_base, kTmemLinear);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  bool aborted = false;
  DevStatus* const st = &sm.status;
  const uint64_t lim = c.wait_ns;

  if (warp >= kWarpTma) {
    rebalance<kLRegOther>();
    if (warp == kWarpTma && lane == 0) {
      // ------------------------------------------------------ TMA producer
      prefetch_tmap(&c.tq);
      prefetch_tmap(&c.tk);
      prefetch_tmap(&c.tv);
      uint32_t used = 0, phase = 0;  // by slot: taken before; parity of the release waited for
      int L = 0;
      const int n_loads = nc * (nh + 2);
      for (int ci = 0, in = 0; L < n_loads; ++L) {
        int s = -1;
        const uint64_t t0 = global_ns();
        for (uint32_t it = 0; s < 0; ++it) {
          for (int i = 0; i < kLSlots && s < 0; ++i)
            if (!((used >> i) & 1u) || mbar_test(&sm.empty[i], (phase >> i) & 1u)) s = i;
          if (s < 0 && (it & 15u) == 15u && global_ns() - t0 > lim) {
            set_status(st, UC_ERR_TIMEOUT, 50);
            aborted = true;
            break;
          }
        }
        if (aborted) break;
        if ((used >> s) & 1u) phase ^= 1u << s;
        used |= 1u << s;
        sm.slot_of[L & 15] = (uint8_t)s;
        uint64_t* bar = &sm.full[L % kLFull];
        const int t = (c0 + ci) * kChunk;
        if (L == c.withhold) {
          // test hook: this tile is never copied
        } else if (in == 0)
          load_tile(sm.slot[s], &c.tk, t, kvh, b, bar);
        else if (in == 2)
          load_tile(sm.slot[s], &c.tv, t, kvh, b, bar);
        else
          load_tile(sm.slot[s], &c.tq, t, kvh * p.group + h0 + (in == 1 ? 0 : in - 2), b, bar);
        if (++in == nh + 2) {
          in = 0;
          ++ci;
        }
      }
      sm.loads = L;
    } else if (warp == kWarpQk) {
      // ---------------------------------------------------------- Q K^T
      const uint32_t lead = elect_one();
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      const uint32_t dhi = (uint32_t)(smem_desc_sw128(0, 16) >> 32);
      const uint32_t row_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.slot[0]), 16);
      for (int ci = 0, t = 0; ci < nc && !aborted; ++ci) {
        uint32_t ks = 0;
        for (int h = 0; h < nh; ++h, ++t) {
          // P of the tile before the last has been read: its slot is free. (Two
          // barriers by tile: the last tile's may complete before this is looked at.)
          if (t > 1 && !dwait_warp(&sm.o_full[t & 1], ((t >> 1) - 1) & 1, st, 58, aborted, lim)) break;
          if (h == 0) {
            const int L = load_k(ci);
            if (!dwait_warp(&sm.full[L % kLFull], (L / kLFull) & 1, st, 54, aborted, lim)) break;
            ks = __shfl_sync(0xffffffffu, (uint32_t)sm.slot_of[L & 15], 0);
            if (valid(ci) < kChunk) zero_rows(sm.slot[ks], valid(ci), lane);
          }
          const int L = load_q(ci, h);
          if (!dwait_warp(&sm.full[L % kLFull], (L / kLFull) & 1, st, 56, aborted, lim)) break;
          const uint32_t qs = __shfl_sync(0xffffffffu, (uint32_t)sm.slot_of[L & 15], 0);
          tc_fence_after();
          issue_q_k(lead, tm + 128 * (t & 1), row_lo + qs * (kTileBytes >> 4), row_lo + ks * (kTileBytes >> 4), dhi,
                    idesc_bf16(128, 128, 0, 0));
          umma_commit_lead(lead, &sm.s_full[t & 1]);
          if (h == nh - 1) umma_commit_lead(lead, &sm.k_done[ci & 1]);
        }
      }
    } else if (warp == kWarpMma) {
      // ------------------------------------------------------ Q S and P V
      const uint32_t lead = elect_one();
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      constexpr uint32_t id_b = idesc_bf16(128, 128, 0, 1);  // B along its rows
      const uint32_t dhi = (uint32_t)(smem_desc_sw128(0, 16) >> 32);
      constexpr uint32_t kStep = kTileBytes >> 4;
      // a slot as an operand along its 128-B rows (q) or across them (v)
      const uint32_t row_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.slot[0]), 16);
      const uint32_t col_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.slot[0]), kTileBytes / 2);
      const uint32_t s_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.s), kTileBytes / 2);
      auto take = [&](int L, int where) -> uint32_t {  // waits for load L; its slot
        dwait_warp(&sm.full[L % kLFull], (L / kLFull) & 1, st, where, aborted, lim);
        return __shfl_sync(0xffffffffu, (uint32_t)sm.slot_of[L & 15], 0);
      };
      for (int ci = 0, t = 0; ci < nc && !aborted; ++ci) {
        uint32_t vs = 0;
        bool gone = valid(ci) == kChunk;  // chunk_go has been given
        for (int h = 0; h < nh; ++h, ++t) {
          const bool last = h == nh - 1;
          const uint32_t qs = take(load_q(ci, h), 56);
          if (h == 0) {
            const uint32_t ks = take(load_k(ci), 60);
            vs = take(load_v(ci), 60);
            if (aborted) break;
            if (valid(ci) < kChunk) zero_rows(sm.slot[vs], valid(ci), lane);
            if (lane == 0) {
              sm.ks[ci & 1] = ks;
              sm.vs[ci & 1] = vs;
              if (gone) mbar_arrive(&sm.chunk_go[ci & 1]);  // the chunk's k and v are there
            }
          }
          if (t > 0 && !dwait_warp(&sm.o_free, (t - 1) & 1, st, 59, aborted, lim)) break;
          // Q S, then P V; a chunk's first tile the other way round, since the
          // state is the last to come
          if (h > 0) {
            tc_fence_after();
            issue_q_s(lead, tm + kColOut, row_lo + qs * kStep, s_lo, dhi, id_b, 0u);
            issue_q_s(lead, tm + kColOut, row_lo + qs * kStep, s_lo - kStep, dhi, id_b, 1u);
            if (last) umma_commit_lead(lead, &sm.s_free);
          }
          if (!dwait_warp(&sm.p_full[t & 1], (t >> 1) & 1, st, 61, aborted, lim)) break;
          if (h == 0 && sm.v_hit[ci & 1] != 0) {
            // (k's zeroed rows are there behind Q K^T, and the update before this one
            // is done where the state's copy is there)
            if (!dwait_warp(&sm.st_ready, ci & 1, st, 57, aborted, lim)) break;
            if (!gone && lane == 0) mbar_arrive(&sm.chunk_go[ci & 1]);
            gone = true;
            if ((ci + 1 < nc || last_state) && !dwait_warp(&sm.kv_done, ci & 1, st, 63, aborted, lim)) break;
            clear_not_finite(sm.slot[vs], lane);
            if (lane == 0) sm.v_odd = 1;
          }
          tc_fence_after();
          if (h > 0) umma_commit_lead(lead, &sm.empty[qs]);  // Q S is issued, and Q K^T was done before P
          issue_p_v(lead, tm + kColOut, tm + 128 * (t & 1), col_lo + vs * kStep, dhi, id_b, h > 0);
          if (h == 0) {
            // the chunk's state is in shared memory, the next scaled in place
            if (!dwait_warp(&sm.st_ready, ci & 1, st, 57, aborted, lim)) break;
            tc_fence_after();
            issue_q_s(lead, tm + kColOut, row_lo + qs * kStep, s_lo, dhi, id_b, 1u);
            issue_q_s(lead, tm + kColOut, row_lo + qs * kStep, s_lo - kStep, dhi, id_b, 1u);
            if (last) umma_commit_lead(lead, &sm.s_free);
            umma_commit_lead(lead, &sm.empty[qs]);
          }
          umma_commit_lead(lead, &sm.o_full[t & 1]);
          if (last) umma_commit_lead(lead, &sm.v_done[ci & 1]);
          // (a last chunk's k rows behind the end were zeroed before its Q K^T)
          if (h == 0 && lane == 0 && !gone) mbar_arrive(&sm.chunk_go[ci & 1]);
        }
      }
    } else if (warp == kWarpSlice) {
      // ---------------------------------------------------- slices' products
      const uint32_t lead = elect_one();
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      constexpr uint32_t id_ab = idesc_bf16(128, 128, 1, 1);  // A and B along their rows
      const uint32_t dhi = (uint32_t)(smem_desc_sw128(0, 16) >> 32);
      const uint32_t col_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.slot[0]), kTileBytes / 2);
      const uint32_t part_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.part[0][0]), kSliceBytes / 2);
      int n = 0;
      for (int ci = 0; ci < (last_state ? nc : nc - 1) && !aborted; ++ci) {
        // (the state is scaled for this chunk before its first slice is formed)
        if (!dwait_warp(&sm.chunk_go[ci & 1], (ci >> 1) & 1, st, 62, aborted, lim)) break;
        const uint32_t ks = __shfl_sync(0xffffffffu, sm.ks[ci & 1], 0), vs = __shfl_sync(0xffffffffu, sm.vs[ci & 1], 0);
        for (int sl = 0; sl < kSlices; ++sl, ++n) {
          const int buf = n & 1;
          if (!dwait_warp(&sm.part_full[buf], (n >> 1) & 1, st, 62, aborted, lim)) break;
          tc_fence_after();
          issue_slice(lead, tm + kColState, col_lo + ks * (kTileBytes >> 4) + 128 * sl,
                      part_lo + buf * (3 * kSliceBytes >> 4), dhi, id_ab);
          umma_commit_lead(lead, &sm.part_free[buf]);
        }
        umma_commit_lead(lead, &sm.kv_done);
        if (!dwait_warp(&sm.kv_done, ci & 1, st, 62, aborted, lim)) break;
        // (two barriers each: the tiles of the next chunk may be done before this is looked at)
        if (!dwait_warp(&sm.k_done[ci & 1], (ci >> 1) & 1, st, 62, aborted, lim)) break;
        if (lane == 0) mbar_arrive(&sm.empty[ks]);
        if (!dwait_warp(&sm.v_done[ci & 1], (ci >> 1) & 1, st, 62, aborted, lim)) break;
        if (lane == 0) mbar_arrive(&sm.empty[vs]);
      }
    }
  } else if (warp >= kWarpState) {
    rebalance<kLRegState>();
    // ---------------------------------------------------------------- state
    const int r = threadIdx.x & 127;  // key channel = TMEM lane
    const uint32_t s_addr = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + kColState;
    if (c.from_start) griddep_wait();
    const size_t row = ((size_t)(b * p.n_kv_heads + kvh) * kHeadDim + r) * kHeadDim;
    const float* src = c.from_start ? c.start + ((size_t)(grun * p.n_kv_heads + kvh) * kHeadDim + r) * kHeadDim
                                    : (p.state_in ? p.state_in + row : nullptr);
#pragma unroll 1
    for (int blk = 0; blk < 4; ++blk) {
      uint32_t w[32];
#pragma unroll
      for (int e = 0; e < 32; e += 4) {
        uint4 x = make_uint4(0, 0, 0, 0);
        if (src) x = *reinterpret_cast<const uint4*>(src + 32 * blk + e);
        w[e] = x.x;
        w[e + 1] = x.y;
        w[e + 2] = x.z;
        w[e + 3] = x.w;
      }
      tmem_st32(s_addr + 32 * blk, w);
    }
    tmem_wait_st();
    auto copy = [&](int blk, int e) {  // eight channels of the row's bf16 copy
      const int chunk16 = 4 * (blk & 1) + e;  // 16 bytes of the row's half
      return reinterpret_cast<uint4*>(sm.s + (blk >> 1) * (kTileBytes / 2) + r * 128 + ((chunk16 ^ (r & 7)) << 4));
    };
    // 32 channels of the state: tensor memory's part and, where there is one, the
    // copy's, scaled by g since it was made (also by 0: an infinity stays one or
    // becomes NaN, as in the recurrence)
    auto whole_state = [&](int blk, uint32_t(&x)[32], bool copied, float g) {
      tmem_ld32(s_addr + 32 * blk, x);
      tmem_wait_ld32(x);
      if (!copied) return;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint4 c = *copy(blk, e);
        const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float a, b;
          f2_unpack(f2_fma(f2_pack(bf16_lo(w[u]), bf16_hi(w[u])), f2_pack(g, g),
                           f2_pack(__uint_as_float(x[8 * e + 2 * u]), __uint_as_float(x[8 * e + 2 * u + 1]))), a, b);
          x[8 * e + 2 * u] = __float_as_uint(a);
          x[8 * e + 2 * u + 1] = __float_as_uint(b);
        }
      }
    };
    int n_slice = 0;
    for (int ci = 0; ci < nc && !aborted; ++ci) {
      const bool update = ci + 1 < nc || last_state;
      const int nv = valid(ci);
      if (ci > 0 && !(dwait_warp(&sm.kv_done, (ci - 1) & 1, st, 66, aborted, lim) &&
                      dwait_warp(&sm.s_free, (ci - 1) & 1, st, 66, aborted, lim)))
        break;
      tc_fence_after();
      const float g = sm.pw[nv];
#pragma unroll 1
      for (int blk = 0; blk < 4; ++blk) {
        uint32_t x[32];
        whole_state(blk, x, ci > 0, sm.pw[kChunk]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t w[4], rest[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            float a = __uint_as_float(x[8 * e + 2 * u]), c = __uint_as_float(x[8 * e + 2 * u + 1]);
            w[u] = pack_bf16(a, c);
            // what rounding leaves (anything finite where the state has overflowed)
            f2_unpack(f2_fma(f2_pack(bf16_lo(w[u]), bf16_hi(w[u])), f2_pack(-1.f, -1.f), f2_pack(a, c)), a, c);
            a = fminf(a, 3e38f);
            c = fminf(c, 3e38f);
            rest[u] = pack_bf16(a, c);
            f2_unpack(f2_mul(f2_pack(a, c), f2_pack(g, g)), a, c);
            x[8 * e + 2 * u] = __float_as_uint(a);
            x[8 * e + 2 * u + 1] = __float_as_uint(c);
          }
          *copy(blk, e) = make_uint4(w[0], w[1], w[2], w[3]);
          *(copy(blk, e) - kTileBytes / 16) = make_uint4(rest[0], rest[1], rest[2], rest[3]);
        }
        if (update) tmem_st32(s_addr + 32 * blk, x);
      }
      tmem_wait_st();
      tc_fence_before();
      fence_proxy_async_smem();
      warp_arrive(&sm.st_ready, lane);
      if (!update) break;
      if (!dwait_warp(&sm.chunk_go[ci & 1], (ci >> 1) & 1, st, 67, aborted, lim)) break;  // V is there
      const uint8_t* v = sm.slot[sm.vs[ci & 1]];
      for (int sl = 0; sl < kSlices; sl += help ? 2 : 1, n_slice += help ? 2 : 1) {
        const int buf = n_slice & 1;
        if (n_slice >= 2 && !dwait_warp(&sm.part_free[buf], ((n_slice >> 1) - 1) & 1, st, 68, aborted, lim)) break;
        decay_slice<kSlice, 128>(v, sm.part[buf], sl, nv, r, [&](int j) { return sm.pw[nv - 1 - j]; });
        fence_proxy_async_smem();
        warp_arrive(&sm.part_full[buf], lane);
      }
    }
    if (last_state && !aborted && (nc == 0 || dwait_warp(&sm.kv_done, (nc - 1) & 1, st, 66, aborted, lim))) {
      tc_fence_after();
      float* dst = p.state_out + row;
#pragma unroll 1
      for (int blk = 0; blk < 4; ++blk) {
        uint32_t x[32];
        whole_state(blk, x, nc > 0, nc > 0 ? sm.pw[valid(nc - 1)] : 0.f);
#pragma unroll
        for (int e = 0; e < 32; e += 4)
          *reinterpret_cast<uint4*>(dst + 32 * blk + e) = make_uint4(x[e], x[e + 1], x[e + 2], x[e + 3]);
      }
    }
    tc_fence_before();
  } else if (warp >= kWarpEpilogue) {
    rebalance<kLRegEpilogue>();
    // ------------------------------------------------------------- epilogue
    const int r = threadIdx.x & 127;  // TMEM lane: token of the tile
    const int half = (warp - kWarpEpilogue) >> 2;  // of the channels
    const uint32_t o_addr = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + kColOut + 64 * half;
    const float f = fmaxf(sm.pw[r + 1], strong ? kLeastScale : 0.f) * p.scale;
    const uint64_t ff = f2_pack(f, f);
    uint4* const turn = sm.turn[warp - kWarpEpilogue];
    for (int ci = 0, t = 0; ci < nc && !aborted; ++ci) {
      const int nv = valid(ci);
      for (int h = 0; h < nh; ++h, ++t) {
        if (!dwait_warp(&sm.o_full[t & 1], (t >> 1) & 1, st, 65, aborted, lim)) break;
        tc_fence_after();
        // o leaves tensor memory before anything else (the next tile's products wait for it)
        uint32_t w[2][16];
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
          uint32_t y[32];
          tmem_ld32(o_addr + 32 * blk, y);
          tmem_wait_ld32(y);
          if (blk == 1) {
            tc_fence_before();
            warp_arrive(&sm.o_free, lane);
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            float y0, y1;
            f2_unpack(f2_mul(f2_pack(__uint_as_float(y[2 * e]), __uint_as_float(y[2 * e + 1])), ff), y0, y1);
            w[blk][e] = pack_bf16(y0, y1);
          }
        }
        if (r >= nv) {  // tokens behind the sequence's end: zeros
#pragma unroll
          for (int e = 0; e < 32; ++e) w[e >> 4][e & 15] = 0u;
        }
        // lane: row 16 i + lane / 2 of the warp's 32, 16 bytes lane mod 2 of each 32
        const int tok = (c0 + ci) * kChunk + 32 * (warp & 3) + (lane >> 1);
        __nv_bfloat16* const o = p.out.at(b, kvh * p.group + h0 + h, tok) + 64 * half + 8 * (lane & 1);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t* x = &w[q >> 1][8 * (q & 1)];
          __syncwarp();
          turn[2 * lane + ((lane >> 2) & 1)] = make_uint4(x[0], x[1], x[2], x[3]);
          turn[2 * lane + (((lane >> 2) & 1) ^ 1)] = make_uint4(x[4], x[5], x[6], x[7]);
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int row = 16 * i + (lane >> 1);
            if (tok + 16 * i < p.n_tok)
              *reinterpret_cast<uint4*>(o + 16 * i * p.out.st + 16 * q) = turn[2 * row + ((lane & 1) ^ ((row >> 2) & 1))];
          }
        }
      }
    }
    tc_fence_before();
  } else {
    rebalance<kLRegP>();
    // -------------------------------------------------------------------- P
    const int x = warp >> 2;          // half of the columns (keys)
    const int r = threadIdx.x & 127;  // TMEM lane: token of the tile
    const int wr = 32 * (warp & 3);   // the warp's first row
    const uint32_t slot0 = tmem + ((uint32_t)wr << 16) + 64 * x;
    // (strong decay only) 1 / a_i
    const float inv_a = strong ? 1.f / fmaxf(sm.pw[r + 1], kLeastScale) : 0.f;
    int n_odd = 0;
    for (int t = 0, ci = 0, h = 0; t < tiles; ++t) {
      if (!dwait_warp(&sm.s_full[t & 1], (t >> 1) & 1, st, 64, aborted, lim)) break;
      tc_fence_after();
      const uint32_t slot = slot0 + 128 * (t & 1);
      // 16 keys at a time, the next ones' loads in flight (P overwrites only
      // columns that are read); keys behind the warp's last row need no load
      uint32_t sr[2][16];
      if (64 * x < wr + 32) tmem_ld16(slot, sr[0]);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int j0 = 64 * x + 16 * q;
        uint32_t(&y)[16] = sr[q & 1];
        tmem_wait_ld16(y);
        if (q < 3 && j0 + 16 < wr + 32) tmem_ld16(slot + 16 * (q + 1), sr[(q + 1) & 1]);
        uint32_t pk[8], pl[8];
        if (j0 >= wr + 32) {
#pragma unroll
          for (int e = 0; e < 8; ++e) pk[e] = pl[e] = 0u;
        } else if (!strong) {
          const ulonglong2* cj = reinterpret_cast<const ulonglong2*>(sm.cj + j0);  // pairs of fp32
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const ulonglong2 w = cj[e];
            float z[4];
            f2_unpack(f2_mul(f2_pack(__uint_as_float(y[4 * e]), __uint_as_float(y[4 * e + 1])), w.x), z[0], z[1]);
            f2_unpack(f2_mul(f2_pack(__uint_as_float(y[4 * e + 2]), __uint_as_float(y[4 * e + 3])), w.y), z[2], z[3]);
            two_parts(z[0], z[1], pk[2 * e], pl[2 * e]);
            two_parts(z[2], z[3], pk[2 * e + 1], pl[2 * e + 1]);
          }
          if (j0 >= wr) {  // keys up to the token (later ones may hold anything)
            const int last = r - j0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const uint32_t mask = (2 * e <= last ? 0xffffu : 0u) | (2 * e + 1 <= last ? 0xffff0000u : 0u);
              pk[e] &= mask;
              pl[e] &= mask;
            }
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float z[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const int back = r - j0 - 2 * e - u;  // tokens since the key
              z[u] = back >= 0 ? __uint_as_float(y[2 * e + u]) * (sm.pw[max(back, 0)] * inv_a) : 0.f;
            }
            two_parts(z[0], z[1], pk[e], pl[e]);
          }
        }
        tmem_st8(slot + 16 * q, pk);
        tmem_st8(slot + 16 * q + 8, pl);
      }
      if (h == 0) {
        const int L = load_v(ci);
        if (!dwait_warp(&sm.full[L % kLFull], (L / kLFull) & 1, st, 60, aborted, lim)) break;
        const bool odd = holds_not_finite(sm.slot[sm.slot_of[L & 15]], valid(ci), threadIdx.x);
        if (lane == 0) reinterpret_cast<uint8_t*>(&sm.v_hit[ci & 1])[warp] = odd;
      }
      tmem_wait_st();
      tc_fence_before();
      warp_arrive(&sm.p_full[t & 1], lane);
      if (++h < nh) continue;
      if (help && (ci + 1 < nc || last_state)) {  // the chunk's odd slices
        if (!dwait_warp(&sm.chunk_go[ci & 1], (ci >> 1) & 1, st, 67, aborted, lim)) break;
        const uint8_t* v = sm.slot[sm.vs[ci & 1]];
        const int nv = valid(ci);
        for (int sl = 1; sl < kSlices; sl += 2, ++n_odd) {
          if (n_odd > 0 && !dwait_warp(&sm.part_free[1], (n_odd - 1) & 1, st, 68, aborted, lim)) break;
          decay_slice<kSlice, 256>(v, sm.part[1], sl, nv, threadIdx.x, [&](int j) { return sm.pw[nv - 1 - j]; });
          fence_proxy_async_smem();
          warp_arrive(&sm.part_full[1], lane);
        }
        if (aborted) break;
      }
      h = 0;
      ++ci;
    }
    tmem_wait_st();
    tc_fence_before();
  }
  __syncthreads();
  if (sm.status.code != 0) drain_cta(sm, c.status, c.withhold, warp);
  if (warp == kWarpMma) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, kTmemLinear);
  }
  if (sm.v_odd) {
    int cta = blockIdx.x;
    asm volatile("" : "+r"(cta));
    spoil_outputs(c, cta, reinterpret_cast<int*>(sm.turn));
  }
}

// A run's own sum: sum_j k_j (gamma^{e-1-j} v_j)^T over its tokens, e its end
// (a sequence's last run needs none). The weights fall towards the run's
// start, so the chunks add up without a rescale: each one's sum in tensor
// memory from zero, in turns of two, and all of them in registers (rounded,
// where the tensor cores cut). Four groups of four warps form the decayed
// values, a quarter chunk each, and hold a quarter of the channels. A pass over
// k and v: about 4000 cycles a chunk (131072 tokens of 4 heads: 57 us, 4.7 TB/s),
// bound by shared memory: at 128 B a cycle the products' operands take 1500, the
// parts' 96 KB 800, the tiles 800. (Barriers per half of a group's quarter, or v
// freed before k: the same.)
constexpr int kLocalRing = 2;  // chunks in flight
constexpr int kQuarter = kChunk / 4;
constexpr uint32_t kQuarterBytes = kQuarter * kHeadDim * 2;
struct LinearLocalSmem {
  uint8_t k[kLocalRing][kTileBytes], v[kLocalRing][kTileBytes];
  uint8_t part[4][3][kQuarterBytes];  // [2 x 64 channels][32 tokens][128 B]
  float pw[kChunk];                   // gamma^n
  uint64_t k_full[kLocalRing], v_full[kLocalRing], empty[kLocalRing];
  uint64_t part_full[4], part_free[4], sum_full[2], sum_free[2], drain;
  uint32_t tmem_base;
  int loads;         // chunks loaded
  DevStatus status;  // as in LinearSmem
};
static_assert(sizeof(LinearLocalSmem) + 1024 <= 232448, "linear attention shared memory");

__global__ void __launch_bounds__(kLThreads, 1) linear_local_kernel(const __grid_constant__ LinearChunkParams c) {
  extern __shared__ uint8_t dyn_smem[];
  LinearLocalSmem& sm = *reinterpret_cast<LinearLocalSmem*>(
      (reinterpret_cast<uintptr_t>(dyn_smem) + 1023) & ~static_cast<uintptr_t>(1023));
  griddep_launch_dependents();
  const LinearParams& p = c.p;
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int kvh = blockIdx.x % p.n_kv_heads, grun = blockIdx.x / p.n_kv_heads;
  const int b = sequence_of(c.plan, p.batch, grun);
  if (grun + 1 == c.plan.run_begin[b + 1]) return;
  const int c0 = (grun - c.plan.run_begin[b]) * c.plan.chunks_per_run;
  const int nc = c.plan.chunks_per_run;  // every chunk of a run before the last is whole
  if (threadIdx.x == 0) {
    for (int s = 0; s < kLocalRing; ++s) {
      mbar_init(&sm.k_full[s], 1);
      mbar_init(&sm.v_full[s], 1);
      mbar_init(&sm.empty[s], 1);
    }
    for (int s = 0; s < 4; ++s) {
      mbar_init(&sm.part_full[s], 4);
      mbar_init(&sm.part_free[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&sm.sum_full[s], 1);
      mbar_init(&sm.sum_free[s], 16);
    }
    mbar_init(&sm.drain, 1);
    fence_barrier_init();
    sm.loads = 0;
    sm.status.code = 0;
  }
  const float2 l2 = p.log2_decay[kvh];
  if (threadIdx.x < kChunk) sm.pw[threadIdx.x] = decay_pow(l2, threadIdx.x);
  if (warp == kWarpMma) tmem_alloc(&sm.tmem_base, 256);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  bool aborted = false;
  DevStatus* const st = &sm.status;
  const uint64_t lim = c.wait_ns;
  if (warp == kWarpTma && lane == 0) {
    prefetch_tmap(&c.tk);
    prefetch_tmap(&c.tv);
    int loaded = 0;
    for (int ci = 0; ci < nc; ++ci) {
      const int s = ci % kLocalRing;
      if (ci >= kLocalRing && !dwait(&sm.empty[s], (ci / kLocalRing - 1) & 1, st, 70, aborted, lim)) break;
      load_tile(sm.v[s], &c.tv, (c0 + ci) * kChunk, kvh, b, &sm.v_full[s]);
      if (ci != c.withhold_sum) load_tile(sm.k[s], &c.tk, (c0 + ci) * kChunk, kvh, b, &sm.k_full[s]);  // (test hook)
      loaded = ci + 1;
    }
    sm.loads = loaded;
  } else if (warp == kWarpMma) {
    const uint32_t lead = elect_one();
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    constexpr uint32_t id_ab = idesc_bf16(128, 128, 1, 1);  // A and B along their rows
    const uint32_t dhi = (uint32_t)(smem_desc_sw128(0, 16) >> 32);
    const uint32_t k_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.k[0]), kTileBytes / 2);
    const uint32_t part_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.part[0][0]), kQuarterBytes / 2);
    for (int ci = 0; ci < nc && !aborted; ++ci) {
      const int s = ci % kLocalRing;
      uint32_t first = 0;
      if (ci > 1 && !dwait_warp(&sm.sum_free[ci & 1], ((ci >> 1) - 1) & 1, st, 77, aborted, lim)) break;
      if (!dwait_warp(&sm.k_full[s], (ci / kLocalRing) & 1, st, 73, aborted, lim)) break;
      for (int g = 0; g < 4; ++g) {
        if (!dwait_warp(&sm.part_full[g], ci & 1, st, 75, aborted, lim)) break;
        tc_fence_after();
#pragma unroll 1
        for (uint32_t u = 0; u < 6; ++u) {  // three parts of two 16-token steps
          const uint32_t step = u & 1;
          issue_ss(lead, tm + 128 * (ci & 1), k_lo + s * (kTileBytes >> 4) + (kQuarter * 128 >> 4) * g + 128 * step,
                   part_lo + (3 * g + (u >> 1)) * (kQuarterBytes >> 4) + 128 * step, dhi, id_ab, first);
          first = 1;
        }
        umma_commit_lead(lead, &sm.part_free[g]);
      }
      umma_commit_lead(lead, &sm.empty[s]);
      umma_commit_lead(lead, &sm.sum_full[ci & 1]);
    }
  } else if (warp < 16) {
    const int g = warp >> 2;
    // a chunk's own sum (32 rows, 32 channels per warp) joins the others in registers
    float sum[32] = {};
    auto fold = [&](int ci) {
      if (!dwait_warp(&sm.sum_full[ci & 1], (ci >> 1) & 1, st, 77, aborted, lim)) return false;
      tc_fence_after();
      uint32_t x[32];
      tmem_ld32(tmem + ((uint32_t)(32 * (warp & 3)) << 16) + 128 * (ci & 1) + 32 * g, x);
      tmem_wait_ld32(x);
#pragma unroll
      for (int e = 0; e < 32; ++e) sum[e] += __uint_as_float(x[e]);
      tc_fence_before();
      warp_arrive(&sm.sum_free[ci & 1], lane);
      return true;
    };
    for (int ci = 0; ci < nc; ++ci) {
      const int s = ci % kLocalRing;
      // gamma^{e - 1 - t} = gamma^{tokens of the run behind this chunk} gamma^{127 - j}
      const float behind = decay_pow(l2, (nc - 1 - ci) * kChunk);
      if (!dwait_warp(&sm.v_full[s], (ci / kLocalRing) & 1, st, 76, aborted, lim)) break;
      if (ci > 0 && !dwait_warp(&sm.part_free[g], (ci - 1) & 1, st, 76, aborted, lim)) break;
      decay_slice<kQuarter, 128>(sm.v[s], sm.part[g], g, kChunk, threadIdx.x & 127,
                                 [&](int j) { return behind * sm.pw[kChunk - 1 - j]; });
      fence_proxy_async_smem();
      warp_arrive(&sm.part_full[g], lane);
      if (ci > 0 && !fold(ci - 1)) break;
    }
    if (!aborted && fold(nc - 1)) {
      float* dst = c.local + ((size_t)(grun * p.n_kv_heads + kvh) * kHeadDim + (threadIdx.x & 127)) * kHeadDim + 32 * g;
#pragma unroll
      for (int e = 0; e < 32; e += 4)
        *reinterpret_cast<float4*>(dst + e) = make_float4(sum[e], sum[e + 1], sum[e + 2], sum[e + 3]);
    }
    tc_fence_before();
  }
  __syncthreads();
  if (sm.status.code != 0) {  // as drain_cta
    if (threadIdx.x == 0) set_status(c.status, sm.status.code, sm.status.detail);
    bool gone = false;
    if (warp == kWarpTma) {
      const int loads = sm.loads;
#pragma unroll 1
      for (int i = max(0, loads - kLocalRing); i < loads; ++i) {
        if (i != c.withhold_sum) dwait_warp(&sm.k_full[i % kLocalRing], (i / kLocalRing) & 1, c.status, 71, gone);
        dwait_warp(&sm.v_full[i % kLocalRing], (i / kLocalRing) & 1, c.status, 71, gone);
      }
    } else if (warp == kWarpMma) {
      umma_commit_lead(elect_one(), &sm.drain);
      dwait_warp(&sm.drain, 0, c.status, 72, gone);
    }
    __syncthreads();
  }
  if (warp == kWarpMma) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 256);
  }
}

// start of every run from the sums of the runs before it, four elements per
// thread: S <- gamma^{tokens of the run} S + local. (A sequence of one run
// starts from its state_in; this copies it where state_out is the same array
// and several CTAs read it.)
constexpr int kJoinThreads = 128;
__global__ void __launch_bounds__(kJoinThreads) linear_join_kernel(const __grid_constant__ LinearChunkParams c) {
  griddep_launch_dependents();
  griddep_wait();
  const LinearParams& p = c.p;
  constexpr int kBlocks = kHeadDim * kHeadDim / 4 / kJoinThreads;
  const int bh = blockIdx.x / kBlocks, b = bh / p.n_kv_heads, kvh = bh % p.n_kv_heads;
  const int first = c.plan.run_begin[b], runs = c.plan.run_begin[b + 1] - first;
  const size_t in = 4 * ((blockIdx.x % kBlocks) * kJoinThreads + threadIdx.x);
  const size_t step = (size_t)p.n_kv_heads * kHeadDim * kHeadDim;
  const size_t at = (size_t)first * step + (size_t)kvh * kHeadDim * kHeadDim + in;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (p.state_in) s = *reinterpret_cast<const float4*>(p.state_in + (size_t)bh * kHeadDim * kHeadDim + in);
  const float g = decay_pow(p.log2_decay[kvh], c.plan.chunks_per_run * kChunk);
  constexpr int kAhead = 8;  // sums in flight
  for (int run0 = 0; run0 < runs; run0 += kAhead) {
    float4 l[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (run0 + u + 1 < runs) l[u] = *reinterpret_cast<const float4*>(c.local + (run0 + u) * step + at);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (run0 + u >= runs) break;
      *reinterpret_cast<float4*>(c.start + (run0 + u) * step + at) = s;
      if (run0 + u + 1 < runs)
        s = make_float4(fmaf(s.x, g, l[u].x), fmaf(s.y, g, l[u].y), fmaf(s.z, g, l[u].z), fmaf(s.w, g, l[u].w));
    }
  }
}

// Zeros for the tokens behind a sequence's last chunk with a valid one (the
// chunk kernel writes those inside it). One CTA per (sequence, query head,
// kZeroRows tokens).
constexpr int kZeroRows = 512;
__global__ void __launch_bounds__(256) linear_zero_kernel(const __grid_constant__ LinearParams p) {
  const int b = blockIdx.z, h = blockIdx.y;
  const int begin = max((int)blockIdx.x * kZeroRows, (p.lengths[b] + kChunk - 1) / kChunk * kChunk);
  const int end = min(p.n_tok, ((int)blockIdx.x + 1) * kZeroRows);
  for (int64_t i = 16ll * begin + threadIdx.x; i < 16ll * end; i += 256)
    *reinterpret_cast<uint4*>(p.out.at(b, h, (int)(i >> 4)) + 8 * (int)(i & 15)) = make_uint4(0, 0, 0, 0);
}

void launch_linear_chunks(const LinearChunkParams& c, cudaStream_t st) {
  constexpr size_t kSmem = sizeof(LinearSmem) + 1024, kLocalSmem = sizeof(LinearLocalSmem) + 1024;
  static std::once_flag once;
  std::call_once(once, [] {
    cudaFuncSetAttribute(linear_chunk_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
    cudaFuncSetAttribute(linear_local_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kLocalSmem);
  });
  const LinearParams& p = c.p;
  bool behind = false;
  for (int b = 0; b < p.batch; ++b) behind |= (p.lengths[b] + kChunk - 1) / kChunk * kChunk < p.n_tok;
  if (behind) {
    linear_zero_kernel<<<dim3((p.n_tok + kZeroRows - 1) / kZeroRows, p.n_q_heads, p.batch), 256, 0, st>>>(p);
    count_launch();
  }
  if (c.plan.several) {
    linear_local_kernel<<<c.plan.runs * p.n_kv_heads, kLThreads, kLocalSmem, st>>>(c);
    count_launch();
  }
  if (c.from_start) {
    launch_maybe_pdl(c.plan.several, linear_join_kernel, p.batch * p.n_kv_heads * (kHeadDim * kHeadDim / 4 / kJoinThreads),
                     kJoinThreads, 0, st, c);
    count_launch();
  }
  launch_maybe_pdl(c.from_start, linear_chunk_kernel, c.plan.runs * p.n_kv_heads * c.plan.head_parts, kLThreads, kSmem, st, c);
  count_launch();
}

}  // namespace uc
