// Attention with a sliding window and first tokens over a cache whose rows may
// be a ring, for few queries: single tokens, drafts, short pieces of a prompt.
//
// Keys and values in reach are read once, by mma.sync warps that hold them in
// registers alone: K rows are B operands of S = Q K^T as they lie in memory
// (16 bytes of a row per lane, the channels of the k steps taken in that order on
// both sides), and S's accumulators are P's A operand of O += P V after the softmax.
// The V operand wants two keys' elements side by side: rows of two keys per lane,
// interleaved by byte permutation, output channels in the order in which they
// come. P enters as two bf16 parts, so outputs carry their own rounding and no
// other; sums and the online softmax are fp32.
//
// A CTA of four warps takes up to 64 query rows (tokens x heads of a KV head, 16
// a warp) and a range of keys; the ranges of a row block go to the CTAs of a
// cluster, which joins them through distributed shared memory, and where that is
// not enough to several clusters, joined by a second kernel.
#include <climits>
#include <cmath>
#include <cstring>
#include <mutex>

#include "args.h"
#include "common.cuh"
#include "internal.h"
#include "window.cuh"

namespace uc {

namespace {

constexpr int kStepWarps = 4;
constexpr int kTileKeys = 16;

struct StepSmem {
  float o[kStepWarps][16][kHeadDim + 4];  // (rows 16 bytes apart in banks)
  float m[kStepWarps][16], l[kStepWarps][16];
};

__device__ __forceinline__ uint32_t rank_addr(const void* local, int rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(local)), "r"(rank));
  return a;
}
__device__ __forceinline__ float ld_rank(uint32_t a) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ float4 ld_rank4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(a)
               : "memory");
  return v;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// RG: warps side by side over a block's rows (16 each); the others take keys.
template <int RG>
__global__ void __launch_bounds__(32 * kStepWarps) window_step_kernel(const __grid_constant__ WindowParams p) {
  constexpr int kKeyWarps = kStepWarps / RG;
  extern __shared__ __align__(16) uint8_t dyn[];
  StepSmem& sm = *reinterpret_cast<StepSmem*>(dyn);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, j = lane & 3;
  const int rank = blockIdx.x % p.cluster;
  int at = blockIdx.x / p.cluster;
  const int split = at % p.splits;
  at /= p.splits;
  const int block = at % p.row_blocks;
  at /= p.row_blocks;
  const int kvh = at % p.n_kv_heads, b = at / p.n_kv_heads;
  const int rg = warp % RG, kw = warp / RG;
  const int rows = p.group * p.n_tok, row0 = block * kWindowRows;
  const WindowSeq s = window_seq(p, b);
  if (threadIdx.x == 0) window_check(p, b);
  // positions of the block's rows that are queries
  const int ta = row0 / p.group, tb = min(min(row0 + kWindowRows, rows) - 1, p.group * s.nq - 1) / p.group;
  WindowKeys keys = {0, 0, 0};
  if (p.group * s.nq > row0) keys = window_keys(p, s, s.first + ta, s.first + tb);
  const int n = keys.count();
  const int base = window_row(p, keys.lo);
  // this warp's 16 rows: r0 + g and r0 + g + 8
  const int r0 = row0 + 16 * rg;
  const int rr[2] = {r0 + g, r0 + g + 8};
  int pos[2];
  uint32_t q[8][4];  // A operands of the 8 k steps
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int t = rr[i] / p.group, h = kvh * p.group + rr[i] % p.group;
    const bool is = rr[i] < rows && t < s.nq;
    pos[i] = is ? s.first + t : INT_MIN;  // (sees nothing)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      uint4 w = make_uint4(0u, 0u, 0u, 0u);
      if (is) w = *reinterpret_cast<const uint4*>(p.q.at(b, h, t) + 32 * c + 8 * j);
      q[2 * c][i] = w.x;
      q[2 * c][2 + i] = w.y;
      q[2 * c + 1][i] = w.z;
      q[2 * c + 1][2 + i] = w.w;
    }
  }
  // (of the warp's queries: a tile of keys up to the first of them and inside the last's window needs no mask)
  const int pfirst = s.first + r0 / p.group, plast = s.first + min(r0 + 15, rows - 1) / p.group;
  const bool active = r0 < rows && r0 / p.group < s.nq;

  float o[16][4];
#pragma unroll
  for (int i = 0; i < 16; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

  const __nv_bfloat16* const kb = p.k.at(b, kvh, 0);
  const __nv_bfloat16* const vb = p.v.at(b, kvh, 0);
  // the cache's row of the i-th key
  auto row_of = [&](int i) {
    int r = i < keys.sinks ? i : base + (i - keys.sinks);
    if (i >= keys.sinks && r >= p.n_rows) r -= p.n_rows - p.n_sink;
    return r;
  };
  uint4 kr[2][4];
  auto load_k = [&](int i0) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int i = i0 + g + 8 * x;
      const uint4* const src = reinterpret_cast<const uint4*>(kb + (int64_t)row_of(min(i, n - 1)) * p.k.st) + j;
#pragma unroll
      for (int c = 0; c < 4; ++c) kr[x][c] = src[4 * c];
    }
  };
  uint4 vr[4][2];
  auto load_v = [&](int i0) {
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int i = i0 + 2 * j + (x & 1) + 8 * (x >> 1);
      const uint4* const src = reinterpret_cast<const uint4*>(vb + (int64_t)row_of(min(i, n - 1)) * p.v.st) + g;
      vr[x][0] = src[0];
      vr[x][1] = src[8];
    }
  };
  // tiles of 16 keys in turn over the splits, the cluster's CTAs and the key warps
  const int stride = kTileKeys * kKeyWarps * p.cluster * p.splits;
  int i0 = kTileKeys * ((split * p.cluster + rank) * kKeyWarps + kw);
  if (!active) i0 = n;
  if (i0 < n) {
    load_k(i0);
    load_v(i0);
  }
  for (; i0 < n; i0 += stride) {
    float x[2][4];
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[y][e] = 0.f;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      mma_bf16(x[0], q[2 * c], kr[0][c].x, kr[0][c].y);
      mma_bf16(x[1], q[2 * c], kr[1][c].x, kr[1][c].y);
      mma_bf16(x[0], q[2 * c + 1], kr[0][c].z, kr[0][c].w);
      mma_bf16(x[1], q[2 * c + 1], kr[1][c].z, kr[1][c].w);
    }
    if (i0 + stride < n) load_k(i0 + stride);
    const int ka = keys.position(i0), kz = keys.position(i0 + kTileKeys - 1);
    const bool whole = i0 + kTileKeys <= n && kz <= pfirst && (plast - ka < p.window || kz < p.n_sink);
    // x[y][e]: row rr[e / 2], key i0 + 8 y + 2 j + e % 2
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[y][e] *= p.scale_log2;
        if (!whole) {
          const int i = i0 + 8 * y + 2 * j + (e & 1);
          if (i >= n || !window_sees(p, pos[e >> 1], keys.position(i))) x[y][e] = -INFINITY;
        }
        top[e >> 1] = fmaxf(top[e >> 1], x[y][e]);
      }
    float old[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
      top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
      old[i] = m[i];
      m[i] = fmaxf(m[i], top[i]);
    }
    if (__any_sync(0xffffffffu, m[0] > old[0] || m[1] > old[1])) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float a = m[i] > old[i] ? ex2_approx(old[i] - m[i]) : 1.f;
        l[i] *= a;
#pragma unroll
        for (int y = 0; y < 16; ++y) {
          o[y][2 * i] *= a;
          o[y][2 * i + 1] *= a;
        }
      }
    }
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float mb = m[i] == -INFINITY ? 0.f : m[i];
        const float a = ex2_approx(x[y][2 * i] - mb), c = ex2_approx(x[y][2 * i + 1] - mb);
        l[i] += a + c;
        const uint32_t w = pack_bf16(a, c);
        hi[2 * y + i] = w;
        lo[2 * y + i] = pack_bf16(a - bf16_lo(w), c - bf16_hi(w));
      }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const uint32_t* const v0 = &vr[0][half].x;
      const uint32_t* const v1 = &vr[1][half].x;
      const uint32_t* const v2 = &vr[2][half].x;
      const uint32_t* const v3 = &vr[3][half].x;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t sel = e & 1 ? 0x7632u : 0x5410u;
        const uint32_t b0 = __byte_perm(v0[e >> 1], v1[e >> 1], sel), b1 = __byte_perm(v2[e >> 1], v3[e >> 1], sel);
        mma_bf16(o[8 * half + e], hi, b0, b1);
        mma_bf16(o[8 * half + e], lo, b0, b1);
      }
    }
    if (i0 + stride < n) load_v(i0 + stride);
  }
  // this warp's part: o[8 half + e][2 i + c]: row g + 8 i, channel 64 half + 16 j + 8 c + e
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
    if (j == 0) {
      sm.m[warp][g + 8 * i] = m[i];
      sm.l[warp][g + 8 * i] = l[i];
    }
#pragma unroll
    for (int y = 0; y < 16; y += 4)
#pragma unroll
      for (int c = 0; c < 2; ++c)
        *reinterpret_cast<float4*>(&sm.o[warp][g + 8 * i][64 * (y >> 3) + 16 * j + 8 * c + (y & 7)]) =
            make_float4(o[y][2 * i + c], o[y + 1][2 * i + c], o[y + 2][2 * i + c], o[y + 3][2 * i + c]);
  }
  cluster_barrier();
  // a warp per row: rows in turn over the cluster's warps
  const int live = min(kWindowRows, rows - row0);
  const int parts = p.cluster * kKeyWarps;  // part c * kKeyWarps + w: warp w * RG + (row / 16) of CTA c
  for (int r = rank + p.cluster * warp; r < live; r += p.cluster * kStepWarps) {
    const int rgr = r >> 4, ri = r & 15;
    auto part_m = [&](int i) {
      return ld_rank(rank_addr(&sm.m[(i % kKeyWarps) * RG + rgr][ri], i / kKeyWarps));
    };
    auto part_l = [&](int i) {
      return ld_rank(rank_addr(&sm.l[(i % kKeyWarps) * RG + rgr][ri], i / kKeyWarps));
    };
    float pm[2], top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int i = lane + 32 * x;
      pm[x] = i < parts ? part_m(i) : -INFINITY;
      top = fmaxf(top, pm[x]);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    const float mb = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int i = lane + 32 * x;
      pm[x] = ex2_approx(pm[x] - mb);
      if (i < parts) sum += pm[x] * part_l(i);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int i = 0; i < parts; ++i) {
      const float w = __shfl_sync(0xffffffffu, i < 32 ? pm[0] : pm[1], i & 31);
      const float4 z = ld_rank4(rank_addr(&sm.o[(i % kKeyWarps) * RG + rgr][ri][4 * lane], i / kKeyWarps));
      y.x += w * z.x;
      y.y += w * z.y;
      y.z += w * z.z;
      y.w += w * z.w;
    }
    const int row = row0 + r, t = row / p.group, h = kvh * p.group + row % p.group;
    if (p.splits == 1) {
      if (t < s.nq)
        window_store_row(p, b, h, t, y, top, sum);
      else
        window_store_row(p, b, h, t, make_float4(0.f, 0.f, 0.f, 0.f), 0.f, 0.f);
    } else {
      // [b, kvh][split][row]: 128 sums, then m and l
      float* const to = p.part + (((int64_t)(b * p.n_kv_heads + kvh) * p.splits + split) * rows + row) * (kHeadDim + 4);
      *reinterpret_cast<float4*>(to + 4 * lane) = y;
      if (lane == 0) *reinterpret_cast<float2*>(to + kHeadDim) = make_float2(top, sum);
    }
  }
  cluster_barrier();  // no CTA leaves while another may still read its shared memory
}

// Rows from the parts of several splits: a warp per row.
__global__ void __launch_bounds__(128) window_join_kernel(const __grid_constant__ WindowParams p) {
  const int lane = threadIdx.x & 31, rows = p.group * p.n_tok;
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int64_t pair = at / rows;
  if (pair >= (int64_t)p.batch * p.n_kv_heads) return;
  const int row = (int)(at - pair * rows), b = (int)(pair / p.n_kv_heads), kvh = (int)(pair % p.n_kv_heads);
  const int t = row / p.group, h = kvh * p.group + row % p.group;
  const int nq = p.n_query ? min(max(p.n_query[b], 0), p.n_tok) : p.n_tok;
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
  float m = -INFINITY, l = 0.f;
  if (t < nq) {
    const int64_t step = (int64_t)rows * (kHeadDim + 4);
    const float* const from = p.part + (pair * p.splits * rows + row) * (kHeadDim + 4);
    for (int i = 0; i < p.splits; ++i) {
      const float2 ml = *reinterpret_cast<const float2*>(from + i * step + kHeadDim);
      const float4 z = *reinterpret_cast<const float4*>(from + i * step + 4 * lane);
      const float top = fmaxf(m, ml.x), mb = top == -INFINITY ? 0.f : top;
      const float a = ex2_approx(m - mb), c = ex2_approx(ml.x - mb);
      y = make_float4(y.x * a + z.x * c, y.y * a + z.y * c, y.z * a + z.z * c, y.w * a + z.w * c);
      l = l * a + ml.y * c;
      m = top;
    }
  }
  window_store_row(p, b, h, t, y, m, l);
}

template <int RG>
void step_launch(const WindowParams& p, cudaStream_t st) {
  static std::once_flag once;
  std::call_once(once, [] {
    cudaFuncSetAttribute(window_step_kernel<RG>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(StepSmem));
    cudaFuncSetAttribute(window_step_kernel<RG>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  });
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.cluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = (unsigned)((int64_t)p.batch * p.n_kv_heads * p.row_blocks * p.splits * p.cluster);
  cfg.blockDim = 32 * kStepWarps;
  cfg.dynamicSmemBytes = sizeof(StepSmem);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaLaunchKernelEx(&cfg, window_step_kernel<RG>, p);
  count_launch();
}

}  // namespace

void launch_window_step(const WindowParams& p, cudaStream_t st) {
  const int rows = std::min(p.group * p.n_tok, kWindowRows);
  if (rows <= 16)
    step_launch<1>(p, st);
  else if (rows <= 32)
    step_launch<2>(p, st);
  else
    step_launch<4>(p, st);
  if (p.splits > 1) launch_window_join(p, st);
}

void launch_window_join(const WindowParams& p, cudaStream_t st) {
  const int64_t all = (int64_t)p.batch * p.n_q_heads * p.n_tok;
  window_join_kernel<<<(unsigned)((all + 3) / 4), 128, 0, st>>>(p);
  count_launch();
}

namespace {

struct WindowPlan {
  bool prompt;
  int row_blocks, cluster, splits;  // (prompt: row_blocks are pairs of Q tiles)
};

// Keys that a block of rows may have in reach.
int64_t most_keys(const uc_window_cache& c, int n_tok, int group) {
  const int64_t tokens = std::min<int64_t>(n_tok, kWindowRows / group + 2);
  return std::min<int64_t>(c.n_rows, (int64_t)c.window + c.n_sink + tokens);
}

WindowPlan plan_window(const uc_window_cache& c, int n_q_heads, int n_tok) {
  WindowPlan w;
  const int group = n_q_heads / c.n_kv_heads;
  const int64_t rows = (int64_t)group * n_tok;
  w.row_blocks = (int)((rows + kWindowRows - 1) / kWindowRows);
  const int64_t items = (int64_t)c.batch * c.n_kv_heads * w.row_blocks;
  w.splits = 1;
  w.prompt = rows > kWindowRows && group <= 128 && c.batch <= kWindowSeqs;
  if (w.prompt) {
    // key ranges of a tile or more where there are too few pairs of Q tiles for the SMs
    const int tokens = 128 / group;
    w.row_blocks = (n_tok + 2 * tokens - 1) / (2 * tokens);
    w.cluster = 1;
    const int64_t all = (int64_t)c.batch * c.n_kv_heads * w.row_blocks;
    const int64_t tiles = (std::min<int64_t>(c.n_rows, (int64_t)c.window + c.n_sink + std::min(n_tok, 2 * tokens)) + 127) / 128;
    w.splits = (int)std::max<int64_t>(1, std::min<int64_t>(num_sms() / all, tiles / 4));
    return w;
  }
  const int rg = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  // CTAs with at least one tile a warp, up to what the SMs hold of them
  const int64_t tiles = (most_keys(c, n_tok, group) + kTileKeys * (kStepWarps / rg) - 1) / (kTileKeys * (kStepWarps / rg));
  const int64_t want = std::max<int64_t>(1, std::min(tiles, 2 * (int64_t)num_sms() / items));
  w.cluster = 1;
  while (2 * w.cluster <= std::min<int64_t>(want, 8)) w.cluster *= 2;
  return w;
}

uc_status check_window_shape(const uc_window_cache& c, int n_q_heads, int n_tok, const char* fn) {
  if (n_q_heads < c.n_kv_heads || n_q_heads % c.n_kv_heads != 0 || n_q_heads > 65535 || n_tok < 1 || n_tok > (1 << 28) ||
      (int64_t)(n_q_heads / c.n_kv_heads) * n_tok > (1 << 30) ||
      (int64_t)c.batch * n_q_heads * n_tok > (1 << 30)) {
    set_error("%s: unsupported shape (batch %d, query heads %d, kv heads %d, tokens %d)", fn, c.batch, n_q_heads,
              c.n_kv_heads, n_tok);
    return UC_ERR_SHAPE;
  }
  return UC_OK;
}

size_t window_bytes(const uc_window_cache& c, int n_q_heads, int n_tok, const WindowPlan& w) {
  if (w.splits == 1) return 256;
  return 256 + (size_t)c.batch * n_q_heads * n_tok * w.splits * (kHeadDim + 4) * sizeof(float);
}

}  // namespace
}  // namespace uc

using namespace uc;

extern "C" {

size_t uc_window_workspace_size(const uc_window_cache* cache, int32_t n_q_heads, int32_t n_tok) {
  UC_TRACE();
  if (cache == nullptr || cache->batch < 1 || cache->batch > 65535 || cache->n_kv_heads < 1 ||
      cache->n_kv_heads > 65535 || cache->n_rows < 1 || cache->n_rows > (1 << 30) || cache->window < 1 ||
      cache->n_sink < 0 || check_window_shape(*cache, n_q_heads, n_tok, "uc_window_workspace_size") != UC_OK)
    return 0;
  return window_bytes(*cache, n_q_heads, n_tok, plan_window(*cache, n_q_heads, n_tok));
}

uc_status uc_window_attend(const uc_window_cache* cache, const uc_rows* q, int32_t n_q_heads, int32_t n_tok,
                           const int32_t* lengths, const int32_t* n_query, const uc_rows* out, float* lse,
                           void* workspace, size_t workspace_bytes, void* stream) {
  UC_TRACE();
  const char* const fn = "uc_window_attend";
  WindowParams p;
  memset(&p, 0, sizeof(p));
  uint64_t nk, nv, nq, no;
  uc_status st = check_window_cache(cache, fn, &p.k, &p.v, &nk, &nv);
  if (st == UC_OK) st = check_window_shape(*cache, n_q_heads, n_tok, fn);
  if (st == UC_OK) st = check_rows(q, fn, "q", cache->batch, n_q_heads, n_tok, &p.q, &nq);
  if (st == UC_OK) st = check_rows(out, fn, "out", cache->batch, n_q_heads, n_tok, &p.out, &no);
  if (st != UC_OK) return st;
  if (lengths == nullptr || !aligned(lengths, 4) || !aligned(n_query, 4) || !aligned(lse, 4)) {
    set_error("uc_window_attend: null or misaligned argument");
    return UC_ERR_ARG;
  }
  const int batch = cache->batch, hkv = cache->n_kv_heads;
  const WindowPlan w = plan_window(*cache, n_q_heads, n_tok);
  st = check_workspace(workspace, workspace_bytes, window_bytes(*cache, n_q_heads, n_tok, w), fn);
  if (st != UC_OK) return st;
  const RowSet ro{&p.out, {batch, n_q_heads, n_tok}, no};
  const RowSet in[3] = {{&p.q, {batch, n_q_heads, n_tok}, nq},
                        {&p.k, {batch, hkv, cache->n_rows}, nk},
                        {&p.v, {batch, hkv, cache->n_rows}, nv}};
  const uint64_t nl = lse ? 4ull * batch * n_q_heads * n_tok : 0, nb = 4ull * batch;
  bool shared = rows_meet(ro, ro) || rows_meet(ro, lengths, nb) || (n_query && rows_meet(ro, n_query, nb)) ||
                (lse && rows_meet(ro, lse, nl)) || overlap(lse, nl, lengths, nb) ||
                overlap(lse, nl, n_query, n_query ? nb : 0);
  for (const RowSet& x : in) shared |= rows_meet(ro, x) || (lse && rows_meet(x, lse, nl));
  if (shared) {
    set_error("uc_window_attend: outputs overlap inputs, each other or themselves");
    return UC_ERR_ARG;
  }
  p.lse = lse;
  p.lengths = lengths;
  p.n_query = n_query;
  p.status = static_cast<DevStatus*>(workspace);
  p.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + 256);
  p.batch = batch;
  p.n_q_heads = n_q_heads;
  p.n_kv_heads = hkv;
  p.group = n_q_heads / hkv;
  p.n_tok = n_tok;
  p.n_rows = cache->n_rows;
  p.window = std::min(cache->window, 1 << 30);  // (more than any row's distance, and no sum passes 32 bits)
  p.n_sink = cache->n_sink;
  p.scale_log2 = (float)(1.4426950408889634074 / std::sqrt((double)UC_HEAD_DIM));
  p.row_blocks = w.row_blocks;
  p.cluster = w.cluster;
  p.splits = w.splits;
  if (!w.prompt) {
    launch_window_step(p, reinterpret_cast<cudaStream_t>(stream));
    return cuda_check(fn);
  }
  WindowPromptParams c;
  memset(&c, 0, sizeof(c));
  c.p = p;
  c.tokens = 128 / p.group;
  st = encode_heads_4d(&c.tq, p.q, n_tok, n_q_heads, batch, p.group, c.tokens);
  const int rest = (cache->n_sink + 15) / 16 * 16 % 128;
  for (int i = 0; i < 2 && st == UC_OK; ++i) {
    const RowsDev& r = i == 0 ? p.k : p.v;
    CUtensorMap* const m = i == 0 ? c.tk : c.tv;
    st = encode_rows_4d(&m[0], r, cache->n_rows, hkv, batch, 128);
    if (st == UC_OK && rest > 0) st = encode_rows_4d(&m[1], r, cache->n_rows, hkv, batch, rest);
  }
  if (st != UC_OK) return st;
  c.wide_out = aligned(p.out.base, 32) && p.out.sb % 16 == 0 && p.out.sh % 16 == 0 && p.out.st % 16 == 0;
  c.wait_ns = wait_limit_ns();
  c.withhold = take_withhold_pos();
  const int64_t items = (int64_t)batch * hkv * w.row_blocks * w.splits;
  const int grid = (int)std::min<int64_t>(items, num_sms());
  const cudaStream_t cs = reinterpret_cast<cudaStream_t>(stream);
  if (items > grid) {
    c.taken = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(workspace) + 128);
    cudaMemsetAsync(c.taken, 0, sizeof(uint32_t), cs);
  }
  launch_window_prompt(c, grid, cs);
  return cuda_check(fn);
}

}  // extern "C"
