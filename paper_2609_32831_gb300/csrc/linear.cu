// Linear attention with a decay for each KV head over a state of constant
// size: per sequence and KV head, with gamma = exp(log_decay) <= 1,
//   S_t = gamma S_{t-1} + k_t v_t^T        (128 x 128, fp32)
//   o_t = S_t^T q_t / sqrt(128)            for every query head of the KV head.
#include <mutex>

#include "common.cuh"
#include "internal.h"

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
  const double gamma = exp2(p.log2_decay[kvh]);
  const float g_hi = (float)gamma, g_lo = (float)(gamma - (double)g_hi);
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

void launch_linear(const LinearParams& p, cudaStream_t st) {
  linear_step_kernel<<<p.batch * p.n_kv_heads * (kHeadDim / kStepCols), 32 * kStepWarps, 0, st>>>(p);
  count_launch();
}

}  // namespace uc
