// Attention with a sliding window and first tokens over a cache whose rows may be a
// ring, for few query rows of a KV head: single tokens, short drafts. (More rows, and
// what plans and joins calls of either kind: plan_window, window_join_kernel.)
//
// Keys and values in reach are read once, 32 keys at a time, by bulk copies into shared
// memory some tiles ahead (rows loaded to registers cost a tile its latency, 2.4K
// cycles; cp.async 1.1K to issue). mma.sync, eight query rows a warp, both products with the keys or channels
// as the 16 rows, so that few query rows waste little: S^T = K Q^T, the channels of the
// k steps in the order of 16-byte pieces on both sides; O^T += V^T P^T with two keys'
// elements brought side by side by byte permutation, the channels in the order in
// which they come, and P^T from S^T's accumulators by a transposition of 8 x 8
// registers. P enters as two bf16 parts, so outputs carry their own rounding and no
// other; sums and the online softmax are fp32.
//
// A CTA takes up to 64 query rows (tokens x heads of a KV head, 8 a warp) and a
// share of the keys, tile by tile over its warps; the shares of a row block go to the
// CTAs of a cluster, which joins them through distributed shared memory, and
// where that is not enough to several clusters, joined by a second kernel.
#include <atomic>
#include <climits>
#include <cmath>
#include <cstring>

#include "args.h"
#include "common.cuh"
#include "internal.h"
#include "window.cuh"

namespace uc {

namespace {

constexpr int kTileKeys = 32;

constexpr int kWarpRows = 8;
constexpr int kStages = 2;
constexpr int kMostWarps = 12;
constexpr int kMostCluster = 8;

struct StepPart {  // of a warp
  float o[kWarpRows][kHeadDim + 4];  // (rows 16 bytes apart in banks)
  float m[kWarpRows], l[kWarpRows];
};
// Tiles of the warps that share keys: 16-byte pieces of K and V rows. (Rows lie 256 bytes
// apart, so that K's reads take two turns and V's four: 190 of a tile's 1000 cycles.)
struct StepRing {
  uint4 k[kStages][kTileKeys][16], v[kStages][kTileKeys][16];
};
// Shared memory of a CTA: barriers; rings, and in their place the parts once the keys are through.
constexpr int kStepHeader = 8 * kStages * 8;
__host__ __device__ constexpr size_t step_smem(int row_warps, int key_warps) {
  const size_t rings = key_warps * sizeof(StepRing), parts = row_warps * key_warps * sizeof(StepPart);
  return kStepHeader + (rings > parts ? rings : parts);
}

__device__ __forceinline__ uint32_t rank_addr(const void* local, int rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(local)), "r"(rank));
  return a;
}
__device__ __forceinline__ float ld_rank(uint32_t a) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ float4 ld_rank4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(a));
  return v;
}
__device__ __forceinline__ int cluster_register_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return (int)r;
}
__device__ __forceinline__ int cluster_register_id() {
  uint32_t r;
  asm("mov.u32 %0, %%clusterid.x;" : "=r"(r));
  return (int)r;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// p.row_warps side by side over a block's rows (8 each) times p.key_warps over its keys.
__global__ void __launch_bounds__(32 * kMostWarps, 1) window_step_kernel(const __grid_constant__ WindowParams p) {
  extern __shared__ __align__(16) uint8_t dyn[];
  uint64_t* const bars = reinterpret_cast<uint64_t*>(dyn);  // [key warp][stage]: a tile has arrived
  StepPart* const sm = reinterpret_cast<StepPart*>(dyn + kStepHeader);
  StepRing* const rings = reinterpret_cast<StepRing*>(dyn + kStepHeader);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, j = lane & 3;
  // (runtime divisions take 100 cycles each: none where a register or a comparison does)
  const int rank = cluster_register_rank();
  int block = cluster_register_id(), split = 0;
  if (p.splits > 1) {
    split = block % p.splits;
    block /= p.splits;
  }
  const int kvh = blockIdx.y, b = blockIdx.z;
  const int kw = p.row_warps == 1 ? warp : warp / p.row_warps, rg = warp - kw * p.row_warps;
  const int rows = p.group * p.n_tok, row0 = block * kWindowRows;
  // token and head of the block's r-th row
  const int t_first = row0 == 0 ? 0 : row0 / p.group, h_first = row0 - t_first * p.group;
  const float per_group = 1.f / (float)p.group;
  auto token_of = [&](int r) { return (int)(((float)(h_first + r) + 0.5f) * per_group); };  // (exact: below 2^17)
  const WindowSeq s = window_seq(p, b);
  if (threadIdx.x == 0) window_check(p, b);
  // positions of the block's rows that are queries
  const int last = min(min(row0 + kWindowRows, rows), p.group * s.nq) - 1 - row0;
  WindowKeys keys = {0, 0, 0};
  if (last >= 0) keys = window_keys(p, s, s.first + t_first, s.first + t_first + token_of(last));
  const int n = keys.count();
  const int base = window_row(p, keys.lo);
  // this warp's rows of the block: as a B operand row g; of S^T's and O^T's accumulators rows 2 j and 2 j + 1
  const int r0 = kWarpRows * rg;
  const bool active = r0 <= last;
  uint4 q[4];
  {
    const int dt = token_of(r0 + g), h = kvh * p.group + h_first + r0 + g - dt * p.group;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      q[c] = make_uint4(0u, 0u, 0u, 0u);
      if (r0 + g <= last) q[c] = *reinterpret_cast<const uint4*>(p.q.at(b, h, t_first + dt) + 32 * c + 8 * j);
    }
  }
  int pos[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    pos[i] = r0 + 2 * j + i <= last ? s.first + t_first + token_of(r0 + 2 * j + i) : INT_MIN;  // (sees nothing)
  // (of the warp's queries: a tile of keys up to the first of them and inside the last's window needs no mask)
  const int pfirst = s.first + t_first + token_of(r0), plast = s.first + t_first + token_of(min(r0 + kWarpRows - 1, last));

  float o[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
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
  // tiles of keys in turn over the splits, the cluster's CTAs and the key warps; the
  // rows of a tile in turn over the warps that share it
  const int stride = kTileKeys * p.key_warps * p.cluster * p.splits;
  int i0 = kTileKeys * ((split * p.cluster + rank) * p.key_warps + kw);
  StepRing& ring = rings[kw];
  uint64_t* const full = bars + kw * kStages;
  if (rg == 0) {
    if (lane < kStages) mbar_init(&full[lane], 1);
    // (rows of V that no copy fills are multiplied by 0)
    for (int x = lane; x < kStages * kTileKeys * 16; x += 32) (&ring.v[0][0][0])[x] = make_uint4(0u, 0u, 0u, 0u);
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  __syncthreads();
  // The copies of a tile: of rows that lie one behind another in the cache, as far as they do. (Where
  // they never do, in token-major caches, 64 copies a tile by this lane bound the kernel: 64 sequences
  // x 4 heads x 4100 keys 233 us instead of 84.)
  const bool dense = p.k.st == kHeadDim && p.v.st == kHeadDim;
  int loads = 0;
  auto copy = [&](int first, int slot) {
    if (first >= n || loads++ == p.withhold) return;
    const int end = min(first + kTileKeys, n);
    mbar_arrive_expect_tx(&full[slot], 2 * (end - first) * kHeadDim * 2);
    for (int i = first; i < end;) {
      const int row = row_of(i);
      const int len = dense ? min(end, i < keys.sinks ? keys.sinks : i + p.n_rows - row) - i : 1;
      bulk_load(&ring.k[slot][i - first][0], kb + (int64_t)row * p.k.st, len * kHeadDim * 2, &full[slot]);
      bulk_load(&ring.v[slot][i - first][0], vb + (int64_t)row * p.v.st, len * kHeadDim * 2, &full[slot]);
      i += len;
    }
  };
  if (rg == 0 && lane == 0)
    for (int x = 0; x < kStages; ++x) copy(i0 + x * stride, x);
  // every warp that shares a tile is through with it: its place is free for another
  auto done = [&]() {
    if (p.row_warps == 1)
      __syncwarp();
    else
      asm volatile("bar.sync %0, %1;" ::"r"(1 + kw), "r"(32 * p.row_warps) : "memory");
  };
  uint32_t parity = 0;
  bool aborted = false;  // a wait ran out: nothing more is copied or computed
  int slot = 0, seen = 0;
  auto next = [&]() {
    done();
    if (rg == 0 && lane == 0 && !aborted) copy(i0 + kStages * stride, slot);
    if (++slot == kStages) {
      slot = 0;
      parity ^= 1u;
    }
    i0 += stride;
  };
  for (; i0 < n; next()) {
    if (!aborted && !mbar_wait(&full[slot], parity, p.status, 100, p.wait_ns)) aborted = true;
    aborted = __any_sync(0xffffffffu, aborted);
    if (aborted) continue;
    ++seen;
    if (!active) continue;
    // x[u]: keys 16 u + g (0, 1) and 16 u + g + 8 (2, 3), rows 2 j (0, 2) and 2 j + 1 (1, 3)
    constexpr int kU = kTileKeys / 16;
    float x[kU][4];
    const int ka = keys.position(i0), kz = keys.position(i0 + kTileKeys - 1);
    const bool whole = i0 + kTileKeys <= n && kz <= pfirst && (plast - ka < p.window || kz < p.n_sink);
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[u][e] = y[e] = 0.f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint4 k0 = ring.k[slot][16 * u + g][4 * c + j], k1 = ring.k[slot][16 * u + g + 8][4 * c + j];
        const uint32_t a0[4] = {k0.x, k1.x, k0.y, k1.y}, a1[4] = {k0.z, k1.z, k0.w, k1.w};
        mma_bf16(x[u], a0, q[c].x, q[c].y);
        mma_bf16(y, a1, q[c].z, q[c].w);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) x[u][e] = (x[u][e] + y[e]) * p.scale_log2;
    }
    if (!whole) {
#pragma unroll
      for (int u = 0; u < kU; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = i0 + 16 * u + g + 8 * (e >> 1);
          if (i >= n || !window_sees(p, pos[e & 1], keys.position(i))) x[u][e] = -INFINITY;
        }
    }
    float old[2], top[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      top[i] = fmaxf(x[0][i], x[0][2 + i]);
#pragma unroll
      for (int u = 1; u < kU; ++u) top[i] = fmaxf(top[i], fmaxf(x[u][i], x[u][2 + i]));
    }
#pragma unroll
    for (int d = 4; d <= 16; d <<= 1) {
      top[0] = fmaxf(top[0], __shfl_xor_sync(0xffffffffu, top[0], d));
      top[1] = fmaxf(top[1], __shfl_xor_sync(0xffffffffu, top[1], d));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      old[i] = m[i];
      m[i] = fmaxf(m[i], top[i]);
    }
    if (__any_sync(0xffffffffu, m[0] > old[0] || m[1] > old[1])) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float a = m[i] > old[i] ? ex2_approx(old[i] - m[i]) : 1.f;
        l[i] *= a;
#pragma unroll
        for (int z = 0; z < 8; ++z) {
          o[z][i] *= a;
          o[z][2 + i] *= a;
        }
      }
    }
    const float mb[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
    uint32_t hi[kU][2], lo[kU][2];
#pragma unroll
    for (int u = 0; u < kU; ++u)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float a = ex2_approx(x[u][2 * k] - mb[0]), c = ex2_approx(x[u][2 * k + 1] - mb[1]);
        l[0] += a;
        l[1] += c;
        const uint32_t w = pack_bf16(a, c);
        hi[u][k] = movmatrix_t(w);
        lo[u][k] = movmatrix_t(pack_bf16(a - bf16_lo(w), c - bf16_hi(w)));
      }
#pragma unroll
    for (int u = 0; u < kU; ++u)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint4 w[4];  // keys 2 j, 2 j + 1, 2 j + 8, 2 j + 9
#pragma unroll
        for (int z = 0; z < 4; ++z) w[z] = ring.v[slot][16 * u + 2 * j + (z & 1) + 8 * (z >> 1)][g + 8 * half];
        const uint32_t* const v0 = &w[0].x;
        const uint32_t* const v1 = &w[1].x;
        const uint32_t* const v2 = &w[2].x;
        const uint32_t* const v3 = &w[3].x;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t a[4] = {__byte_perm(v0[e], v1[e], 0x5410), __byte_perm(v0[e], v1[e], 0x7632),
                                 __byte_perm(v2[e], v3[e], 0x5410), __byte_perm(v2[e], v3[e], 0x7632)};
          mma_bf16(o[4 * half + e], a, hi[u][0], hi[u][1]);
          mma_bf16(o[4 * half + e], a, lo[u][0], lo[u][1]);
        }
      }
  }
  // (the parts lie where the tiles did: all copies have arrived, or are waited for now)
  if (aborted && rg == 0 && lane == 0)
    for (int x = seen; x < loads; ++x)
      if (x != p.withhold) mbar_wait(&full[x % kStages], (x / kStages) & 1, p.status, 101);
  __syncthreads();
  // this warp's part: o[4 half + e][2 c + i]: row 2 j + i, channel 64 half + 8 g + 2 e + c
#pragma unroll
  for (int i = 0; i < 2; ++i) {
#pragma unroll
    for (int d = 4; d <= 16; d <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], d);
    if (g == 0) {
      sm[warp].m[2 * j + i] = m[i];
      sm[warp].l[2 * j + i] = l[i];
    }
#pragma unroll
    for (int z = 0; z < 8; z += 2)
      *reinterpret_cast<float4*>(&sm[warp].o[2 * j + i][64 * (z >> 2) + 8 * g + 2 * (z & 3)]) =
          make_float4(o[z][i], o[z][2 + i], o[z + 1][i], o[z + 1][2 + i]);
  }
  // a warp per row: first the CTA's own parts, in place of the first one, then the cluster's
  const int live = min(kWindowRows, rows - row0), warps = p.row_warps * p.key_warps;
  if (p.key_warps > 1) {
    __syncthreads();
    for (int r = warp; r < live; r += warps) {
      StepPart* const part = sm + r / kWarpRows;
      const int ri = r % kWarpRows;
      float top = -INFINITY;
      for (int w = 0; w < p.key_warps; ++w) top = fmaxf(top, part[w * p.row_warps].m[ri]);
      const float mb = top == -INFINITY ? 0.f : top;
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
      float sum = 0.f;
#pragma unroll 4
      for (int w = 0; w < p.key_warps; ++w) {
        const StepPart& from = part[w * p.row_warps];
        const float a = ex2_approx(from.m[ri] - mb);
        const float4 z = *reinterpret_cast<const float4*>(&from.o[ri][4 * lane]);
        sum += a * from.l[ri];
        y = make_float4(y.x + a * z.x, y.y + a * z.y, y.z + a * z.z, y.w + a * z.w);
      }
      *reinterpret_cast<float4*>(&part->o[ri][4 * lane]) = y;
      __syncwarp();
      if (lane == 0) {
        part->m[ri] = top;
        part->l[ri] = sum;
      }
    }
  }
  cluster_barrier();
  for (int r = rank + p.cluster * warp; r < live; r += p.cluster * warps) {
    const int ri = r % kWarpRows;
    const StepPart* const part = sm + r / kWarpRows;
    float top = -INFINITY, sum = 0.f;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    // all loads before the first use
    float pm[kMostCluster], pl[kMostCluster];
    float4 z[kMostCluster];
#pragma unroll
    for (int c = 0; c < kMostCluster; ++c) {
      pm[c] = -INFINITY;
      pl[c] = 0.f;
      z[c] = y;
      if (c < p.cluster) {
        pm[c] = ld_rank(rank_addr(&part->m[ri], c));
        pl[c] = ld_rank(rank_addr(&part->l[ri], c));
        z[c] = ld_rank4(rank_addr(&part->o[ri][4 * lane], c));
      }
    }
#pragma unroll
    for (int c = 0; c < kMostCluster; ++c) top = fmaxf(top, pm[c]);
    const float mb = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int c = 0; c < kMostCluster; ++c) {
      const float a = ex2_approx(pm[c] - mb);
      sum += a * pl[c];
      y = make_float4(y.x + a * z[c].x, y.y + a * z[c].y, y.z + a * z[c].z, y.w + a * z[c].w);
    }
    const int dt = token_of(r), t = t_first + dt, row = row0 + r, h = kvh * p.group + h_first + r - dt * p.group;
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

}  // namespace

void launch_window_step(const WindowParams& p, cudaStream_t st) {
  static std::atomic<uint64_t> set{0};
  allow_smem(window_step_kernel, step_smem(1, 7), &set);
  const int warps = p.row_warps * p.key_warps;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.cluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((int64_t)p.row_blocks * p.splits * p.cluster), (unsigned)p.n_kv_heads, (unsigned)p.batch);
  cfg.blockDim = 32 * warps;
  cfg.dynamicSmemBytes = step_smem(p.row_warps, p.key_warps);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaLaunchKernelEx(&cfg, window_step_kernel, p);
  count_launch();
  if (p.splits > 1) launch_window_join(p, st);
}

void launch_window_join(const WindowParams& p, cudaStream_t st) {
  const int64_t all = (int64_t)p.batch * p.n_q_heads * p.n_tok;
  window_join_kernel<<<(unsigned)((all + 3) / 4), 128, 0, st>>>(p);
  count_launch();
}

namespace {

constexpr int kQTileRows = 128;  // query rows of a prompt's tile
constexpr int64_t kSmBytes = 228 << 10;  // of shared memory

struct WindowPlan {
  bool prompt;
  int row_blocks, cluster, splits, row_warps, key_warps;  // (prompt: row_blocks are pairs of Q tiles)
};

// Keys that a block of rows may have in reach.
int64_t most_keys(const uc_window_cache& c, int n_tok, int group) {
  const int64_t tokens = std::min<int64_t>(n_tok, kWindowRows / group + 2);
  return std::min<int64_t>(c.n_rows, (int64_t)c.window + c.n_sink + tokens);
}

// Steps: keys in tiles over the warps of a cluster of up to 8 CTAs. The size that the
// SMs are through with first, with a CTA's start and end as long as kStart tiles of a
// warp; where even 8 leave a warp many tiles and SMs idle, several clusters and a join.
// *turns: tiles that a warp takes one after the other, over the rounds of CTAs.
WindowPlan plan_step(const uc_window_cache& c, int64_t rows, int group, int n_tok, int64_t* turns) {
  constexpr int64_t kStart = 6;
  WindowPlan w;
  w.prompt = false;
  w.splits = 1;
  w.row_blocks = (int)((rows + kWindowRows - 1) / kWindowRows);
  const int64_t items = (int64_t)c.batch * c.n_kv_heads * w.row_blocks;
  const int64_t tiles = (most_keys(c, n_tok, group) + kTileKeys - 1) / kTileKeys;
  w.row_warps = (int)std::min<int64_t>((rows + kWarpRows - 1) / kWarpRows, kWindowRows / kWarpRows);
  w.key_warps = w.row_warps == 1 && 16 * items <= num_sms() ? 7 : w.row_warps == 1 ? 3 : w.row_warps <= 5 ? 2 : 1;
  const int64_t ctas = std::min<int64_t>(kSmBytes / ((int64_t)step_smem(w.row_warps, w.key_warps) + 1024),
                                         kMostWarps / (w.row_warps * w.key_warps));
  const int64_t slots = ctas * num_sms();
  int64_t least = INT64_MAX, per = 0;
  for (int n = 1; n <= kMostCluster; ++n) {
    const int64_t k = (tiles + n * w.key_warps - 1) / (n * w.key_warps), rounds = (items * n + slots - 1) / slots;
    if (rounds * (kStart + k) < least) {
      least = rounds * (kStart + k);
      w.cluster = n;
      per = k;
      *turns = rounds * k;
    }
  }
  if (per > 2 * kStart)
    w.splits = (int)std::max<int64_t>(1, std::min<int64_t>(slots / (items * w.cluster), per / kStart));
  return w;
}

// Up to 8 query rows of a KV head go step by step: keys and values are read at 93 % of
// the copy rate. More rows wait for a warp's products and softmax there (64 sequences of
// 35 rows over 4100 keys: 312 us, 109 on the tensor cores), unless there are few keys as well
// (8 sequences of 14 rows over 1030 keys: 12 us instead of 17, with P in one part there). More than
// kWindowSeqs sequences go step by step whatever their rows (257 of 40 rows over 2052 keys: 325 us, 256 on
// the tensor cores 128).
WindowPlan plan_window(const uc_window_cache& c, int n_q_heads, int n_tok) {
  const int group = n_q_heads / c.n_kv_heads;
  const int64_t rows = (int64_t)group * n_tok;
  if (rows <= 2 * kWarpRows || group > kQTileRows || c.batch > kWindowSeqs) {
    int64_t turns = 0;
    const WindowPlan w = plan_step(c, rows, group, n_tok, &turns);
    if (rows <= kWarpRows || turns <= 4 || group > kQTileRows || c.batch > kWindowSeqs) return w;
  }
  // Pairs of Q tiles; ranges of key tiles where these are too few for the SMs, an item's
  // start and end and the join as long as kItem and kJoin tiles.
  constexpr int64_t kItem = 3, kJoin = 3;
  WindowPlan w;
  w.prompt = true;
  w.cluster = w.row_warps = w.key_warps = 1;
  const int tokens = kQTileRows / group;
  w.row_blocks = (n_tok + 2 * tokens - 1) / (2 * tokens);
  const int64_t all = (int64_t)c.batch * c.n_kv_heads * w.row_blocks;
  const int64_t tiles = (std::min<int64_t>(c.n_rows, (int64_t)c.window + c.n_sink + std::min(n_tok, 2 * tokens)) + 127) / 128;
  int64_t least = INT64_MAX;
  w.splits = 1;
  for (int64_t r = 1; r <= std::min<int64_t>(32, std::max<int64_t>(1, tiles / 2)) && (r == 1 || all < 2 * num_sms()); ++r) {
    const int64_t cost = (all * r + num_sms() - 1) / num_sms() * (kItem + (tiles + r - 1) / r) + (r > 1 ? kJoin : 0);
    if (cost < least) {
      least = cost;
      w.splits = (int)r;
    }
  }
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
  const uc_window_cache cut = within_rows(*cache);
  return window_bytes(cut, n_q_heads, n_tok, plan_window(cut, n_q_heads, n_tok));
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
  const uc_window_cache cut = within_rows(*cache);
  cache = &cut;
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
  p.row_warps = w.row_warps;
  p.key_warps = w.key_warps;
  p.wait_ns = wait_limit_ns();
  p.withhold = take_withhold_pos();
  if (!w.prompt) {
    launch_window_step(p, reinterpret_cast<cudaStream_t>(stream));
    return cuda_check(fn);
  }
  WindowPromptParams c;
  memset(&c, 0, sizeof(c));
  c.p = p;
  c.tokens = kQTileRows / p.group;
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
  c.two_parts = (int64_t)p.group * n_tok <= kQTileRows;
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
