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
// partial sums over a warp's rows meet in shared memory.
constexpr int kStepCols = 32;
constexpr int kStepWarps = 8;
constexpr int kStepRows = kHeadDim / kStepWarps;
constexpr int kStepHeads = 8;  // query heads reduced at a time

__global__ void __launch_bounds__(32 * kStepWarps) linear_step_kernel(const __grid_constant__ LinearParams p) {
  __shared__ float qs[kStepHeads][kHeadDim];
  __shared__ float part[kStepHeads][kStepWarps][kStepCols];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int kSlices = kHeadDim / kStepCols;
  const int bh = blockIdx.x / kSlices, slice = blockIdx.x % kSlices;
  const int b = bh / p.n_kv_heads, kvh = bh % p.n_kv_heads;
  const int col = slice * kStepCols + lane;
  const int n = p.lengths[b];
  // gamma as two fp32 parts: rounded to one, a decay that remembers thousands
  // of tokens would drift by their number times 2^-25
  const float g_hi = p.decay[kvh].x, g_lo = p.decay[kvh].y;
  float s[kStepRows];
  const size_t at = ((size_t)bh * kHeadDim + warp * kStepRows) * kHeadDim + col;
#pragma unroll
  for (int r = 0; r < kStepRows; ++r) s[r] = p.state_in ? p.state_in[at + (size_t)r * kHeadDim] : 0.f;
  for (int t = 0; t < p.n_tok; ++t) {
    if (t < n) {
      const __nv_bfloat16* kr = p.k.at(b, kvh, t);
      const float v = __bfloat162float(p.v.at(b, kvh, t)[col]);
#pragma unroll
      for (int r = 0; r < kStepRows; ++r) s[r] = fmaf(s[r], g_hi, fmaf(s[r], g_lo, __bfloat162float(kr[warp * kStepRows + r]) * v));
    }
    for (int h0 = 0; h0 < p.group; h0 += kStepHeads) {
      const int nh = min(kStepHeads, p.group - h0);
      __syncthreads();
      for (int i = threadIdx.x; i < nh * kHeadDim; i += blockDim.x)
        qs[i / kHeadDim][i % kHeadDim] =
            t < n ? __bfloat162float(p.q.at(b, kvh * p.group + h0 + i / kHeadDim, t)[i % kHeadDim]) : 0.f;
      __syncthreads();
      for (int h = 0; h < nh; ++h) {
        float o = 0.f;
#pragma unroll
        for (int r = 0; r < kStepRows; ++r) o = fmaf(qs[h][warp * kStepRows + r], s[r], o);
        part[h][warp][lane] = o;
      }
      __syncthreads();
      for (int i = threadIdx.x; i < nh * kStepCols; i += blockDim.x) {
        float o = 0.f;
#pragma unroll
        for (int w = 0; w < kStepWarps; ++w) o += part[i / kStepCols][w][i % kStepCols];
        // a token behind the sequence's end has no output: zero
        p.out.at(b, kvh * p.group + h0 + i / kStepCols, t)[slice * kStepCols + i % kStepCols] =
            __float2bfloat16_rn(t < n ? o * p.scale : 0.f);
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
//   o_i  = (gamma^{i+1} S^T q_i + sum_{j <= i} gamma^{i-j} (q_i . k_j) v_j) / sqrt(128)
//   S'   = gamma^nv S + sum_j k_j (gamma^{nv-1-j} v_j)^T
// so a chunk costs three 128^3 products per query head (Q K^T, Q S, P V) and
// one per KV head for the state. Bound by HBM: 64 KB of q and o per head and
// chunk against 3 x 512 cycles of the tensor pipe.
//
// One CTA per (sequence, KV head, run of chunks, part of its query heads):
//   warp 8   TMA producer: k and v tiles per chunk, a q tile per head, two slots of each
//   warp 9   issues every tcgen05.mma
//   warp 10  zeroes the k and v rows behind the sequence's end in its last
//            chunk (they may hold NaN, and 0 x NaN is not 0)
//   WG0, WG1 (warps 0-7) halves of the columns of every product: the decay mask on Q K^T (P,
//            bf16, back to tensor memory), the epilogue, the decayed values
//            of the state's update and the state itself, which stays in their
//            registers in fp32 (64 columns of one key channel per thread).
// The jobs of a run are its tiles (chunk, head) in order and, after a chunk's
// last tile, the update of the state. Q K^T of the next tile is issued before
// the current one's other products.
//
// Roundings to bf16: P and the copy of S that Q multiplies (each about as
// large as the output's own rounding), and none of the state's path: the
// decayed values enter as two bf16 parts (v gamma^n to 2^-17), the update
// accumulates in fp32.
constexpr int kLThreads = 384;
constexpr int kLRegCompute = 216;  // 256 x 216 + 128 x 56 registers <= 384 x 168
constexpr int kLRegOther = 56;
static_assert(256 * kLRegCompute + 128 * kLRegOther <= kLThreads * 168, "register split");
constexpr uint32_t kTmemLinear = 512;
constexpr uint32_t kColState = 256;  // O1 = Q S
constexpr uint32_t kColOut = 384;    // O2 = P V; the S slots are columns 0 and 128
constexpr uint32_t kTileBytes = kChunk * kHeadDim * 2;

struct LinearSmem {
  uint8_t k[2][kTileBytes];  // [2 x 64 channels][128 tokens][128 B], 128B swizzle; V becomes the decayed values' hi part
  uint8_t v[2][kTileBytes];
  uint8_t q[2][kTileBytes];  // the slot of a chunk's last tile then takes the lo part
  uint8_t s[kTileBytes];     // the chunk's state, bf16 [2 x 64 value channels][128 key channels][128 B]
  float pw[kChunk + 4];      // gamma^n
  float cf[32];              // gamma^{31 - n}
  uint64_t k_full[2], v_full[2], kv_empty[2], q_full[2], q_empty[2];
  uint64_t s_full[2], p_full[2], o_full, o_free, vt_full, st_ready, last_issued, fixed;
  uint32_t tmem_base;
};
static_assert(sizeof(LinearSmem) + 1024 <= 232448, "linear attention shared memory");

// gamma^n, n >= 0, to fp32 rounding: the exponent n log2(gamma) is formed from
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

// D (+)= A B over 128 rows of both operands in shared memory, K (tokens or key
// channels) along the rows of B: A K-major (q) or along its rows too (k).
template <int KK, int ACC>
__device__ __forceinline__ void issue_q_s_step(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t id) {
  umma_ss_lead<(KK < 4 ? 2 * KK : 1024 + 2 * (KK - 4)), 128 * KK, ACC>(lead, d, a, b, hi, id);
}
__device__ __forceinline__ void issue_q_s(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t id) {
  issue_q_s_step<0, 0>(lead, d, a, b, hi, id);
  issue_q_s_step<1, 1>(lead, d, a, b, hi, id);
  issue_q_s_step<2, 1>(lead, d, a, b, hi, id);
  issue_q_s_step<3, 1>(lead, d, a, b, hi, id);
  issue_q_s_step<4, 1>(lead, d, a, b, hi, id);
  issue_q_s_step<5, 1>(lead, d, a, b, hi, id);
  issue_q_s_step<6, 1>(lead, d, a, b, hi, id);
  issue_q_s_step<7, 1>(lead, d, a, b, hi, id);
}
template <int ACC0>
__device__ __forceinline__ void issue_k_v(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t id) {
  umma_ss_lead<0, 0, ACC0>(lead, d, a, b, hi, id);
  umma_ss_lead<128, 128, 1>(lead, d, a, b, hi, id);
  umma_ss_lead<256, 256, 1>(lead, d, a, b, hi, id);
  umma_ss_lead<384, 384, 1>(lead, d, a, b, hi, id);
  umma_ss_lead<512, 512, 1>(lead, d, a, b, hi, id);
  umma_ss_lead<640, 640, 1>(lead, d, a, b, hi, id);
  umma_ss_lead<768, 768, 1>(lead, d, a, b, hi, id);
  umma_ss_lead<896, 896, 1>(lead, d, a, b, hi, id);
}
// O2 = P V: P of keys 0-63 in the slot's columns 0-31, of keys 64-127 in 64-95
// (each warpgroup's P lies in the columns that it alone read).
__device__ __forceinline__ void issue_p_v(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t id) {
  umma_ts_lead<0>(lead, d, a, b, hi, id, 0u);
  umma_ts_lead<1>(lead, d, a, b, hi, id, 1u);
  umma_ts_lead<2>(lead, d, a, b, hi, id, 1u);
  umma_ts_lead<3>(lead, d, a, b, hi, id, 1u);
  umma_ts_lead<4>(lead, d, a + 32, b, hi, id, 1u);
  umma_ts_lead<5>(lead, d, a + 32, b, hi, id, 1u);
  umma_ts_lead<6>(lead, d, a + 32, b, hi, id, 1u);
  umma_ts_lead<7>(lead, d, a + 32, b, hi, id, 1u);
}

// The decayed values of a chunk as two bf16 parts: hi over V in place, lo into
// `lo`, by `threads` threads. Row j's weight w(j), 0 from row nv on (whatever
// the row holds).
template <typename W>
__device__ __forceinline__ void decay_values(uint8_t* v, uint8_t* lo, int nv, int thread, int threads, const W& weight) {
#pragma unroll 2
  for (int i = thread; i < (int)kTileBytes / 16; i += threads) {
    const int j = (i >> 3) & (kChunk - 1);
    uint4* at = reinterpret_cast<uint4*>(v) + i;
    uint4 h = make_uint4(0, 0, 0, 0), l = h;
    if (j < nv) {
      const float w = weight(j);
      const uint4 x = *at;
      const uint32_t in[4] = {x.x, x.y, x.z, x.w};
      uint32_t hi[4], rest[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float a = bf16_lo(in[e]) * w, b = bf16_hi(in[e]) * w;
        hi[e] = pack_bf16(a, b);
        rest[e] = pack_bf16(a - bf16_lo(hi[e]), b - bf16_hi(hi[e]));
      }
      h = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      l = make_uint4(rest[0], rest[1], rest[2], rest[3]);
    }
    *at = h;
    reinterpret_cast<uint4*>(lo)[i] = l;
  }
  __syncwarp();
}

// Zeroes rows nv .. 127 of a tile, by one warp.
__device__ __forceinline__ void zero_rows(uint8_t* tile, int nv, int lane) {
  for (int half = 0; half < 2; ++half)
    for (int i = nv * 8 + lane; i < kChunk * 8; i += 32)
      reinterpret_cast<uint4*>(tile + half * (kTileBytes / 2))[i] = make_uint4(0, 0, 0, 0);
}

__global__ void __launch_bounds__(kLThreads, 1) linear_chunk_kernel(const __grid_constant__ LinearChunkParams c) {
  extern __shared__ uint8_t dyn_smem[];
  LinearSmem& sm = *reinterpret_cast<LinearSmem*>(
      (reinterpret_cast<uintptr_t>(dyn_smem) + 1023) & ~static_cast<uintptr_t>(1023));
  const LinearParams& p = c.p;
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int part = blockIdx.x % c.plan.head_parts;
  const int run = blockIdx.x / c.plan.head_parts % c.plan.runs;
  const int bh = blockIdx.x / (c.plan.head_parts * c.plan.runs);
  const int b = bh / p.n_kv_heads, kvh = bh % p.n_kv_heads;
  const int h0 = part * c.plan.heads_per_part;
  const int nh = min(c.plan.heads_per_part, p.group - h0);
  const int len = p.lengths[b];
  const int c0 = run * c.plan.chunks_per_run;
  const int n_all = (len + kChunk - 1) / kChunk;  // chunks with a valid token
  const int nc = max(0, min(c.plan.chunks_per_run, n_all - c0));
  // the state behind the last chunk is needed where this launch writes it
  const bool last_state = !c.plan.two_pass;
  auto valid = [&](int ci) { return min(kChunk, len - (c0 + ci) * kChunk); };

  if (threadIdx.x == 0) {
    for (int s = 0; s < 2; ++s) {
      mbar_init(&sm.k_full[s], 1);
      mbar_init(&sm.v_full[s], 1);
      mbar_init(&sm.kv_empty[s], 1);
      mbar_init(&sm.q_full[s], 1);
      mbar_init(&sm.q_empty[s], 1);
      mbar_init(&sm.s_full[s], 1);
      mbar_init(&sm.p_full[s], 256);
    }
    mbar_init(&sm.o_full, 1);
    mbar_init(&sm.o_free, 256);
    mbar_init(&sm.vt_full, 256);
    mbar_init(&sm.st_ready, 256);
    mbar_init(&sm.last_issued, 1);
    mbar_init(&sm.fixed, 32);
    fence_barrier_init();
  }
  if (threadIdx.x <= kChunk) {
    const float w = decay_pow(p.log2_decay[kvh], threadIdx.x);
    sm.pw[threadIdx.x] = w;
    if (threadIdx.x < 32) sm.cf[31 - threadIdx.x] = w;
  }
  if (warp == 9) tmem_alloc(&sm.tmem_base, kTmemLinear);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  bool aborted = false;
  DevStatus* const st = c.status;
  const uint64_t lim = c.wait_ns;

  if (warp >= 8) {
    setmaxnreg_dec<kLRegOther>();
    if (warp == 8 && lane == 0) {
      // ------------------------------------------------------ TMA producer
      prefetch_tmap(&c.tq);
      prefetch_tmap(&c.tk);
      prefetch_tmap(&c.tv);
      int ti = 0, loaded = 0;
      for (int ci = 0; ci < nc && !aborted; ++ci) {
        const int s = ci & 1, t0 = (c0 + ci) * kChunk;
        if (ci >= 2 && !dwait(&sm.kv_empty[s], ((ci >> 1) - 1) & 1, st, 50, aborted, lim)) break;
        load_tile(sm.k[s], &c.tk, t0, kvh, b, &sm.k_full[s]);
        load_tile(sm.v[s], &c.tv, t0, kvh, b, &sm.v_full[s]);
        loaded = ci + 1;
        if (loaded == nc) mbar_arrive(&sm.last_issued);
        for (int h = 0; h < nh; ++h, ++ti) {
          const int qs = ti & 1;
          if (ti >= 2 && !dwait(&sm.q_empty[qs], ((ti >> 1) - 1) & 1, st, 51, aborted, lim)) break;
          load_tile(sm.q[qs], &c.tq, t0, kvh * p.group + h0 + h, b, &sm.q_full[qs]);
        }
      }
      if (aborted) {
        // no copy may land in shared memory that is no longer this CTA's
        bool gone = false;
        for (int i = max(0, loaded - 2); i < loaded; ++i) {
          dwait(&sm.k_full[i & 1], (i >> 1) & 1, st, 52, gone, lim);
          dwait(&sm.v_full[i & 1], (i >> 1) & 1, st, 52, gone, lim);
        }
        for (int i = max(0, ti - 2); i < ti; ++i) dwait(&sm.q_full[i & 1], (i >> 1) & 1, st, 52, gone, lim);
      }
    } else if (warp == 10) {
      // ------------------------------------- rows behind the sequence's end
      if (nc > 0 && valid(nc - 1) < kChunk) {
        const int s = (nc - 1) & 1, ph = ((nc - 1) >> 1) & 1, nv = valid(nc - 1);
        // (once the last copies are issued, the slots' current phase is theirs)
        if (dwait_warp(&sm.last_issued, 0, st, 53, aborted, lim) &&
            dwait_warp(&sm.k_full[s], ph, st, 53, aborted, lim) && dwait_warp(&sm.v_full[s], ph, st, 53, aborted, lim)) {
          zero_rows(sm.k[s], nv, lane);
          zero_rows(sm.v[s], nv, lane);
          fence_proxy_async_smem();
          mbar_arrive(&sm.fixed);
        }
      }
    } else if (warp == 9) {
      // -------------------------------------------------------- MMA issuer
      const uint32_t lead = elect_one();
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      constexpr uint32_t id_qk = idesc_bf16(128, 128, 0, 0);
      constexpr uint32_t id_b = idesc_bf16(128, 128, 0, 1);   // B along its rows
      constexpr uint32_t id_ab = idesc_bf16(128, 128, 1, 1);  // A and B along their rows
      const uint32_t dhi = (uint32_t)(smem_desc_sw128(0, 16) >> 32);
      constexpr uint32_t kStep = kTileBytes >> 4;
      const uint32_t q_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.q[0]), 16);
      const uint32_t k_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.k[0]), 16);
      const uint32_t kt_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.k[0]), kTileBytes / 2);
      const uint32_t v_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.v[0]), kTileBytes / 2);
      const uint32_t s_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.s), kTileBytes / 2);
      const uint32_t lq_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.q[0]), kTileBytes / 2);
      // Q K^T of tile (ci, h), which is job n and tile ti of the run
      auto issue_scores = [&](int n, int ti, int ci, int h) -> bool {
        if (h == 0) {
          if (!dwait_warp(&sm.k_full[ci & 1], (ci >> 1) & 1, st, 54, aborted, lim)) return false;
          if (ci == nc - 1 && valid(ci) < kChunk && !dwait_warp(&sm.fixed, 0, st, 55, aborted, lim)) return false;
        }
        if (!dwait_warp(&sm.q_full[ti & 1], (ti >> 1) & 1, st, 56, aborted, lim)) return false;
        tc_fence_after();
        issue_qk<0>(lead, tm + 128 * (n & 1), q_lo + (ti & 1) * kStep, k_lo + (ci & 1) * kStep, dhi, id_qk);
        umma_commit_lead(lead, &sm.s_full[n & 1]);
        return true;
      };
      int n = 0, ti = 0;
      bool ok = nc > 0 && issue_scores(0, 0, 0, 0);
      for (int ci = 0; ci < nc && ok; ++ci) {
        const bool update = ci + 1 < nc || last_state;
        for (int h = 0; h < nh && ok; ++h, ++n, ++ti) {
          const bool last = h == nh - 1;
          ok = false;
          if (h == 0) {
            // the chunk's state is in shared memory, the update's sums are read
            if (!dwait_warp(&sm.st_ready, ci & 1, st, 57, aborted, lim)) break;
          } else if (!dwait_warp(&sm.o_full, (ti - 1) & 1, st, 58, aborted, lim)) {
            break;  // (the other S slot's P is consumed)
          }
          if (!last && !issue_scores(n + 1, ti + 1, ci, h + 1)) break;
          if (ti > 0 && !dwait_warp(&sm.o_free, (ti - 1) & 1, st, 59, aborted, lim)) break;
          tc_fence_after();
          issue_q_s(lead, tm + kColState, q_lo + (ti & 1) * kStep, s_lo, dhi, id_b);
          if (!(last && update)) umma_commit_lead(lead, &sm.q_empty[ti & 1]);
          if (h == 0 && !dwait_warp(&sm.v_full[ci & 1], (ci >> 1) & 1, st, 60, aborted, lim)) break;
          if (!dwait_warp(&sm.p_full[ti & 1], (ti >> 1) & 1, st, 61, aborted, lim)) break;
          tc_fence_after();
          issue_p_v(lead, tm + kColOut, tm + 128 * (n & 1), v_lo + (ci & 1) * kStep, dhi, id_b);
          umma_commit_lead(lead, &sm.o_full);
          ok = true;
        }
        if (!ok) break;
        if (update) {
          ok = false;
          if (!dwait_warp(&sm.o_full, (ti - 1) & 1, st, 62, aborted, lim)) break;
          if (ci + 1 < nc && !issue_scores(n + 1, ti, ci + 1, 0)) break;
          if (!dwait_warp(&sm.vt_full, ci & 1, st, 63, aborted, lim)) break;
          tc_fence_after();
          const uint32_t d = tm + 128 * (n & 1), a = kt_lo + (ci & 1) * kStep;
          issue_k_v<0>(lead, d, a, v_lo + (ci & 1) * kStep, dhi, id_ab);
          issue_k_v<1>(lead, d, a, lq_lo + ((ti - 1) & 1) * kStep, dhi, id_ab);
          umma_commit_lead(lead, &sm.s_full[n & 1]);
          umma_commit_lead(lead, &sm.kv_empty[ci & 1]);
          umma_commit_lead(lead, &sm.q_empty[(ti - 1) & 1]);
          ++n;
          ok = true;
        }
      }
    }
  } else {
    setmaxnreg_inc<kLRegCompute>();
    // -------------------------------------------------------------- compute
    const int x = warp >> 2;          // half of the columns
    const int r = threadIdx.x & 127;  // TMEM lane: token of the tile, or key channel of the state
    const int wr = 32 * (warp & 3);   // the warp's first row
    const uint32_t lane_off = (uint32_t)wr << 16;
    const int tid = threadIdx.x;
    // state row r (key channel), value channels 64 x .. 64 x + 63
    float sreg[64];
    {
      if (c.plan.two_pass) griddep_wait();
      const float* src = c.plan.two_pass ? c.start + ((size_t)run * p.batch * p.n_kv_heads + bh) * kHeadDim * kHeadDim
                                         : (p.state_in ? p.state_in + (size_t)bh * kHeadDim * kHeadDim : nullptr);
#pragma unroll
      for (int e = 0; e < 64; e += 4) {
        float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
        if (src) w = *reinterpret_cast<const float4*>(src + (size_t)r * kHeadDim + 64 * x + e);
        sreg[e] = w.x;
        sreg[e + 1] = w.y;
        sreg[e + 2] = w.z;
        sreg[e + 3] = w.w;
      }
    }
    auto store_state = [&]() {  // bf16 copy for Q S
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint4 w = make_uint4(pack_bf16(sreg[8 * e], sreg[8 * e + 1]), pack_bf16(sreg[8 * e + 2], sreg[8 * e + 3]),
                                   pack_bf16(sreg[8 * e + 4], sreg[8 * e + 5]), pack_bf16(sreg[8 * e + 6], sreg[8 * e + 7]));
        *reinterpret_cast<uint4*>(sm.s + x * (kTileBytes / 2) + r * 128 + ((e ^ (r & 7)) << 4)) = w;
      }
      fence_proxy_async_smem();
      mbar_arrive(&sm.st_ready);
    };
    if (nc > 0) store_state();
    // P of job n, tile ti: gamma^{i-j} (q_i . k_j) for j <= i, 32 columns at a time
    auto scores = [&](int n, int ti) -> bool {
      if (!dwait_warp(&sm.s_full[n & 1], (n >> 1) & 1, st, 64, aborted, lim)) return false;
      tc_fence_after();
      const uint32_t slot = tmem + lane_off + 128 * (n & 1) + 64 * x;
      uint32_t pk[2][16];
#pragma unroll
      for (int blk = 0; blk < 2; ++blk) {
        const int j0 = 64 * x + 32 * blk;
        if (j0 > wr) {  // above the diagonal
#pragma unroll
          for (int e = 0; e < 16; ++e) pk[blk][e] = 0u;
          continue;
        }
        uint32_t sr[32];
        tmem_ld32(slot + 32 * blk, sr);
        tmem_wait_ld();
        if (j0 < wr) {
          const float rowf = sm.pw[r - j0 - 31];
#pragma unroll
          for (int e = 0; e < 16; ++e)
            pk[blk][e] = pack_bf16(__uint_as_float(sr[2 * e]) * (sm.cf[2 * e] * rowf),
                                   __uint_as_float(sr[2 * e + 1]) * (sm.cf[2 * e + 1] * rowf));
        } else {
          // the diagonal block: lane i, column j (masked entries may hold anything)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float a = 2 * e <= lane ? __uint_as_float(sr[2 * e]) * sm.pw[max(0, lane - 2 * e)] : 0.f;
            const float bb = 2 * e + 1 <= lane ? __uint_as_float(sr[2 * e + 1]) * sm.pw[max(0, lane - 2 * e - 1)] : 0.f;
            pk[blk][e] = pack_bf16(a, bb);
          }
        }
      }
      tmem_st16(slot, pk[0]);
      tmem_st16(slot + 16, pk[1]);
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(&sm.p_full[ti & 1]);
      return true;
    };
    // o of tile ti = (ci, h)
    auto epilogue = [&](int ti, int ci, int h) -> bool {
      if (!dwait_warp(&sm.o_full, ti & 1, st, 65, aborted, lim)) return false;
      tc_fence_after();
      const int nv = valid(ci), t = (c0 + ci) * kChunk + r;
      const float f1 = sm.pw[r + 1] * p.scale, f2 = p.scale;
      __nv_bfloat16* o = t < p.n_tok ? p.out.at(b, kvh * p.group + h0 + h, t) + 64 * x : nullptr;
      uint32_t a[2][32], d[2][32];
#pragma unroll
      for (int blk = 0; blk < 2; ++blk) {
        tmem_ld32(tmem + lane_off + kColState + 64 * x + 32 * blk, a[blk]);
        tmem_ld32(tmem + lane_off + kColOut + 64 * x + 32 * blk, d[blk]);
      }
      tmem_wait_ld();
      tc_fence_before();
      mbar_arrive(&sm.o_free);
      if (o != nullptr) {
#pragma unroll
        for (int u8 = 0; u8 < 8; ++u8) {
          const int blk = u8 >> 2, e = 8 * (u8 & 3);
          uint32_t w[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int i = e + 2 * u;
            const float y0 = fmaf(__uint_as_float(a[blk][i]), f1, __uint_as_float(d[blk][i]) * f2);
            const float y1 = fmaf(__uint_as_float(a[blk][i + 1]), f1, __uint_as_float(d[blk][i + 1]) * f2);
            w[u] = r < nv ? pack_bf16(y0, y1) : 0u;
          }
          *reinterpret_cast<uint4*>(o + 32 * blk + e) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
      __syncwarp();
      return true;
    };
    int n = 0, ti = 0;
    bool ok = true;
    for (int ci = 0; ci < nc && ok; ++ci) {
      const bool update = ci + 1 < nc || last_state;
      for (int h = 0; h < nh && ok; ++h, ++n, ++ti) {
        ok = scores(n, ti);
        if (ok && h > 0) ok = epilogue(ti - 1, ci, h - 1);
      }
      if (!ok) break;
      if (update) {
        const int s = ci & 1, nv = valid(ci);
        // the chunk's products are complete: V and the last q tile's slot are free to be written
        ok = dwait_warp(&sm.o_full, (ti - 1) & 1, st, 66, aborted, lim) &&
             dwait_warp(&sm.v_full[s], (ci >> 1) & 1, st, 67, aborted, lim);
        if (!ok) break;
        decay_values(sm.v[s], sm.q[(ti - 1) & 1], nv, tid, 256, [&](int j) { return sm.pw[nv - 1 - j]; });
        fence_proxy_async_smem();
        mbar_arrive(&sm.vt_full);
        ok = epilogue(ti - 1, ci, nh - 1) && dwait_warp(&sm.s_full[n & 1], (n >> 1) & 1, st, 68, aborted, lim);
        if (!ok) break;
        tc_fence_after();
        const float g = sm.pw[nv];
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
          uint32_t kv[32];
          tmem_ld32(tmem + lane_off + 128 * (n & 1) + 64 * x + 32 * blk, kv);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e) sreg[32 * blk + e] = fmaf(sreg[32 * blk + e], g, __uint_as_float(kv[e]));
        }
        tc_fence_before();
        ++n;
        store_state();
      } else {
        ok = epilogue(ti - 1, ci, nh - 1);
      }
    }
    if (last_state && !aborted) {
      float* dst = p.state_out + ((size_t)bh * kHeadDim + r) * kHeadDim + 64 * x;
#pragma unroll
      for (int e = 0; e < 64; e += 4)
        *reinterpret_cast<float4*>(dst + e) = make_float4(sreg[e], sreg[e + 1], sreg[e + 2], sreg[e + 3]);
    }
    // tokens of this run in chunks behind the sequence's end: zeros
    const int z0 = (c0 + nc) * kChunk, z1 = min(p.n_tok, (c0 + c.plan.chunks_per_run) * kChunk);
    for (int64_t i = tid; i < (int64_t)(z1 - z0) * nh * (kHeadDim / 8); i += 256) {
      const int e = (int)(i % (kHeadDim / 8)), row = (int)(i / (kHeadDim / 8));
      *reinterpret_cast<uint4*>(p.out.at(b, kvh * p.group + h0 + row % nh, z0 + row / nh) + 8 * e) =
          make_uint4(0, 0, 0, 0);
    }
    tc_fence_before();
  }
  __syncthreads();
  if (warp == 9) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, kTmemLinear);
  }
}

// A run's own sum: sum_j k_j (gamma^{e-1-j} v_j)^T over its tokens, e its end.
// The weights fall towards the run's start, so the chunks accumulate in tensor
// memory without a rescale.
struct LinearLocalSmem {
  uint8_t k[2][kTileBytes], v[2][kTileBytes], lo[2][kTileBytes];
  float pw[kChunk];  // gamma^n
  uint64_t k_full[2], v_full[2], empty[2], vt_full[2], done, last_issued, fixed;
  uint32_t tmem_base;
};
static_assert(sizeof(LinearLocalSmem) + 1024 <= 232448, "linear attention shared memory");

__global__ void __launch_bounds__(kLThreads, 1) linear_local_kernel(const __grid_constant__ LinearChunkParams c) {
  extern __shared__ uint8_t dyn_smem[];
  LinearLocalSmem& sm = *reinterpret_cast<LinearLocalSmem*>(
      (reinterpret_cast<uintptr_t>(dyn_smem) + 1023) & ~static_cast<uintptr_t>(1023));
  griddep_launch_dependents();
  const LinearParams& p = c.p;
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int run = blockIdx.x % c.plan.runs, bh = blockIdx.x / c.plan.runs;
  const int b = bh / p.n_kv_heads, kvh = bh % p.n_kv_heads;
  const int len = p.lengths[b];
  const int c0 = run * c.plan.chunks_per_run;
  const int nc = max(0, min(c.plan.chunks_per_run, (len + kChunk - 1) / kChunk - c0));
  auto valid = [&](int ci) { return min(kChunk, len - (c0 + ci) * kChunk); };
  if (threadIdx.x == 0) {
    for (int s = 0; s < 2; ++s) {
      mbar_init(&sm.k_full[s], 1);
      mbar_init(&sm.v_full[s], 1);
      mbar_init(&sm.empty[s], 1);
      mbar_init(&sm.vt_full[s], 256);
    }
    mbar_init(&sm.done, 1);
    mbar_init(&sm.last_issued, 1);
    mbar_init(&sm.fixed, 32);
    fence_barrier_init();
  }
  if (threadIdx.x < kChunk) sm.pw[threadIdx.x] = decay_pow(p.log2_decay[kvh], threadIdx.x);
  if (warp == 9) tmem_alloc(&sm.tmem_base, 128);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  bool aborted = false;
  DevStatus* const st = c.status;
  const uint64_t lim = c.wait_ns;
  if (warp == 8 && lane == 0) {
    prefetch_tmap(&c.tk);
    prefetch_tmap(&c.tv);
    int loaded = 0;
    for (int ci = 0; ci < nc; ++ci) {
      const int s = ci & 1;
      if (ci >= 2 && !dwait(&sm.empty[s], ((ci >> 1) - 1) & 1, st, 70, aborted, lim)) break;
      load_tile(sm.k[s], &c.tk, (c0 + ci) * kChunk, kvh, b, &sm.k_full[s]);
      load_tile(sm.v[s], &c.tv, (c0 + ci) * kChunk, kvh, b, &sm.v_full[s]);
      loaded = ci + 1;
      if (loaded == nc) mbar_arrive(&sm.last_issued);
    }
    if (aborted) {
      bool gone = false;
      for (int i = max(0, loaded - 2); i < loaded; ++i) {
        dwait(&sm.k_full[i & 1], (i >> 1) & 1, st, 71, gone, lim);
        dwait(&sm.v_full[i & 1], (i >> 1) & 1, st, 71, gone, lim);
      }
    }
  } else if (warp == 10) {
    if (nc > 0 && valid(nc - 1) < kChunk) {
      const int s = (nc - 1) & 1;
      if (dwait_warp(&sm.last_issued, 0, st, 72, aborted, lim) &&
          dwait_warp(&sm.k_full[s], ((nc - 1) >> 1) & 1, st, 72, aborted, lim)) {
        zero_rows(sm.k[s], valid(nc - 1), lane);
        fence_proxy_async_smem();
        mbar_arrive(&sm.fixed);
      }
    }
  } else if (warp == 9) {
    const uint32_t lead = elect_one();
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    constexpr uint32_t id_ab = idesc_bf16(128, 128, 1, 1);
    const uint32_t dhi = (uint32_t)(smem_desc_sw128(0, 16) >> 32);
    constexpr uint32_t kStep = kTileBytes >> 4;
    const uint32_t k_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.k[0]), kTileBytes / 2);
    const uint32_t v_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.v[0]), kTileBytes / 2);
    const uint32_t l_lo = (uint32_t)smem_desc_sw128(smem_u32(sm.lo[0]), kTileBytes / 2);
    for (int ci = 0; ci < nc; ++ci) {
      const int s = ci & 1;
      if (!dwait_warp(&sm.k_full[s], (ci >> 1) & 1, st, 73, aborted, lim)) break;
      if (ci == nc - 1 && valid(ci) < kChunk && !dwait_warp(&sm.fixed, 0, st, 74, aborted, lim)) break;
      if (!dwait_warp(&sm.vt_full[s], (ci >> 1) & 1, st, 75, aborted, lim)) break;
      tc_fence_after();
      if (ci == 0)
        issue_k_v<0>(lead, tm, k_lo + s * kStep, v_lo + s * kStep, dhi, id_ab);
      else
        issue_k_v<1>(lead, tm, k_lo + s * kStep, v_lo + s * kStep, dhi, id_ab);
      issue_k_v<1>(lead, tm, k_lo + s * kStep, l_lo + s * kStep, dhi, id_ab);
      umma_commit_lead(lead, &sm.empty[s]);
    }
    umma_commit_lead(lead, &sm.done);
  } else if (warp < 8) {
    const int x = warp >> 2, r = threadIdx.x & 127;
    const int end = min(len, (c0 + c.plan.chunks_per_run) * kChunk);  // the run's last token + 1
    for (int ci = 0; ci < nc; ++ci) {
      const int s = ci & 1, nv = valid(ci);
      // gamma^{end - 1 - t} = gamma^{tokens of the run behind this chunk} gamma^{nv - 1 - j}
      const float behind = decay_pow(p.log2_decay[kvh], end - ((c0 + ci) * kChunk + nv));
      // (the slot's copy is complete only after the products of chunk ci - 2)
      if (!dwait_warp(&sm.v_full[s], (ci >> 1) & 1, st, 76, aborted, lim)) break;
      decay_values(sm.v[s], sm.lo[s], nv, threadIdx.x, 256, [&](int j) { return behind * sm.pw[nv - 1 - j]; });
      fence_proxy_async_smem();
      mbar_arrive(&sm.vt_full[s]);
    }
    float* dst = c.local + (((size_t)run * p.batch * p.n_kv_heads + bh) * kHeadDim + r) * kHeadDim + 64 * x;
    if (nc > 0 && dwait_warp(&sm.done, 0, st, 77, aborted, 2 * lim)) {
      tc_fence_after();
#pragma unroll
      for (int blk = 0; blk < 2; ++blk) {
        uint32_t kv[32];
        tmem_ld32(tmem + ((uint32_t)(32 * (warp & 3)) << 16) + 64 * x + 32 * blk, kv);
        tmem_wait_ld();
#pragma unroll
        for (int e = 0; e < 32; e += 4)
          *reinterpret_cast<uint4*>(dst + 32 * blk + e) = make_uint4(kv[e], kv[e + 1], kv[e + 2], kv[e + 3]);
      }
    } else if (nc == 0) {
      for (int e = 0; e < 64; e += 4) *reinterpret_cast<float4*>(dst + e) = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    tc_fence_before();
  }
  __syncthreads();
  if (warp == 9) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 128);
  }
}

// start[run] and the final state from the runs' own sums, four elements per
// thread: S <- gamma^{tokens of the run} S + local[run].
constexpr int kJoinThreads = 128;
__global__ void __launch_bounds__(kJoinThreads) linear_join_kernel(const __grid_constant__ LinearChunkParams c) {
  griddep_wait();
  griddep_launch_dependents();
  const LinearParams& p = c.p;
  constexpr int kBlocks = kHeadDim * kHeadDim / 4 / kJoinThreads;
  const int bh = blockIdx.x / kBlocks;
  const size_t at = (size_t)bh * kHeadDim * kHeadDim + 4 * ((blockIdx.x % kBlocks) * kJoinThreads + threadIdx.x);
  const size_t step = (size_t)p.batch * p.n_kv_heads * kHeadDim * kHeadDim;
  const int len = p.lengths[bh / p.n_kv_heads];
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (p.state_in) s = *reinterpret_cast<const float4*>(p.state_in + at);
  const int run_tok = c.plan.chunks_per_run * kChunk;
  const float whole = decay_pow(p.log2_decay[bh % p.n_kv_heads], run_tok);
  for (int run = 0; run < c.plan.runs; ++run) {
    const int n = min(run_tok, max(0, len - run * run_tok));
    *reinterpret_cast<float4*>(c.start + run * step + at) = s;
    if (n == 0) continue;
    const float g = n == run_tok ? whole : decay_pow(p.log2_decay[bh % p.n_kv_heads], n);
    const float4 l = *reinterpret_cast<const float4*>(c.local + run * step + at);
    s = make_float4(fmaf(s.x, g, l.x), fmaf(s.y, g, l.y), fmaf(s.z, g, l.z), fmaf(s.w, g, l.w));
  }
  *reinterpret_cast<float4*>(p.state_out + at) = s;
}

void launch_linear_chunks(const LinearChunkParams& c, cudaStream_t st) {
  constexpr size_t kSmem = sizeof(LinearSmem) + 1024, kLocalSmem = sizeof(LinearLocalSmem) + 1024;
  static std::once_flag once;
  std::call_once(once, [] {
    cudaFuncSetAttribute(linear_chunk_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
    cudaFuncSetAttribute(linear_local_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kLocalSmem);
  });
  const int pairs = c.p.batch * c.p.n_kv_heads;
  if (c.plan.two_pass) {
    linear_local_kernel<<<pairs * c.plan.runs, kLThreads, kLocalSmem, st>>>(c);
    count_launch();
    launch_maybe_pdl(true, linear_join_kernel, pairs * (kHeadDim * kHeadDim / 4 / kJoinThreads), kJoinThreads, 0, st, c);
    count_launch();
  }
  launch_maybe_pdl(c.plan.two_pass, linear_chunk_kernel, pairs * c.plan.runs * c.plan.head_parts, kLThreads, kSmem, st, c);
  count_launch();
}

}  // namespace uc
