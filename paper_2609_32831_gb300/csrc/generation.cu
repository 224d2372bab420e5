// C-ABI entry points of generation beside the segment cache: linear attention
// over a constant-size state, beam selection, and the reordering of caches
// and states. Argument validation and launches; nothing here allocates.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>

#include "args.h"
#include "common.cuh"
#include "internal.h"

namespace uc {
namespace {

float2 two_floats(double x) {
  const float hi = (float)x;
  return make_float2(hi, std::isfinite(hi) ? (float)(x - (double)hi) : 0.f);
}

}  // namespace
}  // namespace uc

using namespace uc;

extern "C" {

// ------------------------------------------------------- linear attention
// States of runs that a plan may ask for (64 KB each, twice): the workspace's bound.
constexpr int64_t kMaxLinearSums = 640;

// Decode-shaped calls take the recurrence token by token.
static bool linear_steps(int n_q_heads, int n_kv_heads, int n_tok) {
  return n_tok <= UC_MAX_QTOKENS;
}

// How prompts are cut: over query heads (each part forms the state on its own)
// and over tokens (a pass over k and v before, for the states that the runs
// start from). Costs in clocks of a CTA, from measured launches: a tile of one
// head and chunk, a chunk's update of the state (beside its tiles, a chain that
// takes kChain), a CTA's start and end; the same for the pass before.
static LinearPlan plan_linear(int batch, int n_q_heads, int n_kv_heads, const int32_t* lengths) {
  constexpr double kTile = 4300, kUpdate = 3900, kChain = 11500, kCta = 9000, kSumChunk = 4000, kSumCta = 14000;
  const int g = n_q_heads / n_kv_heads, sms = num_sms();
  int64_t chunks = 0;
  int longest = 1;
  auto chunks_of = [](int n) { return (n + kChunk - 1) / kChunk; };
  for (int b = 0; b < batch; ++b) {
    chunks += chunks_of(lengths[b]);
    longest = std::max(longest, chunks_of(lengths[b]));
  }
  LinearPlan best;
  memset(&best, 0, sizeof(best));
  double least = 0;
  for (int per = 1; per <= g; ++per) {
    const int parts = (g + per - 1) / per;
    if (per > 1 && parts == (g + per - 2) / (per - 1)) continue;  // as many parts as before, less even
    const double chunk = std::max(kChain, kUpdate + per * kTile);
    int last_cpr = 0;
    for (int rounds = 0; rounds <= 4; ++rounds) {
      // whole sequences, or runs that fill so many rounds of CTAs
      int cpr = longest;
      if (rounds > 0) {
        const int64_t want = (int64_t)rounds * sms / ((int64_t)n_kv_heads * parts);
        if (want <= batch) continue;
        cpr = (int)std::max<int64_t>(1, (chunks + want - 1) / want);
        // (sequences' ends leave runs short: raise it until the rounds hold them)
        for (;; ++cpr) {
          int64_t n = 0;
          for (int b = 0; b < batch; ++b) n += std::max(1, (chunks_of(lengths[b]) + cpr - 1) / cpr);
          if (n <= want || cpr >= longest) break;
        }
      }
      if (cpr == last_cpr) continue;
      last_cpr = cpr;
      int64_t n = 0;
      bool several = false;
      double total = 0, most = 0;
      for (int b = 0; b < batch; ++b) {
        const int nb = chunks_of(lengths[b]), r = std::max(1, (nb + cpr - 1) / cpr);
        n += r;
        several |= r > 1;
        total += (double)n_kv_heads * parts * (r * kCta + nb * chunk);
        most = std::max(most, kCta + std::min(cpr, nb) * chunk);
      }
      if (n * n_kv_heads * parts > INT32_MAX) continue;
      if (several && n * n_kv_heads > kMaxLinearSums) continue;
      const double ctas = (double)n * n_kv_heads * parts;
      // (unequal ones fill in behind each other)
      double cost = std::min(std::ceil(ctas / sms) * most, std::max(1.15 * total / sms, most));
      if (several) {
        const double sums = (double)(n - batch) * n_kv_heads;
        cost += std::ceil(sums / sms) * (kSumCta + cpr * kSumChunk);
      }
      if (least == 0 || cost < least) {
        least = cost;
        best.chunks_per_run = cpr;
        best.head_parts = parts;
        best.heads_per_part = per;
        best.several = several;
      }
    }
  }
  for (int b = 0; b < batch; ++b)
    best.run_begin[b + 1] =
        best.run_begin[b] + std::max(1, (chunks_of(lengths[b]) + best.chunks_per_run - 1) / best.chunks_per_run);
  best.runs = best.run_begin[batch];
  return best;
}

// Bytes of `states` pairs of run states (own sum, start) behind the header.
static size_t linear_bytes(uint64_t states) { return 256 + 2 * states * UC_HEAD_DIM * UC_HEAD_DIM * sizeof(float); }

size_t uc_linear_workspace_size(int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t n_tok) {
  UC_TRACE();
  if (batch < 1 || n_kv_heads < 1 || n_q_heads < n_kv_heads || n_tok < 1) return 0;
  if (linear_steps(n_q_heads, n_kv_heads, n_tok)) return 256;
  // whatever the lengths: every chunk a run of its own, as far as plans go
  const uint64_t pairs = (uint64_t)batch * n_kv_heads, chunks = (n_tok + kChunk - 1) / kChunk;
  return linear_bytes(std::max(pairs, std::min(pairs * chunks, (uint64_t)kMaxLinearSums)));
}

uc_status uc_linear_attend(const uc_rows* q, const uc_rows* k, const uc_rows* v, int32_t batch, int32_t n_q_heads,
                           int32_t n_kv_heads, int32_t n_tok, const int32_t* lengths, const float* log_decay,
                           const float* state_in, float* state_out, const uc_rows* out, void* workspace,
                           size_t workspace_bytes, void* stream) {
  UC_TRACE();
  if (batch < 1 || batch > UC_MAX_BATCH || n_kv_heads < 1 || n_kv_heads > UC_MAX_LINEAR_HEADS ||
      n_q_heads < n_kv_heads || n_q_heads % n_kv_heads != 0 || n_q_heads > 65535 || n_tok < 1 || n_tok > (1 << 28)) {
    set_error("uc_linear_attend: unsupported shape (batch %d, query heads %d, kv heads %d, tokens %d)", batch,
              n_q_heads, n_kv_heads, n_tok);
    return UC_ERR_SHAPE;
  }
  LinearParams p;
  memset(&p, 0, sizeof(p));
  uint64_t nq, nk, nv, no;
  const char* const fn = "uc_linear_attend";
  uc_status st = check_rows(q, fn, "q", batch, n_q_heads, n_tok, &p.q, &nq);
  if (st == UC_OK) st = check_rows(k, fn, "k", batch, n_kv_heads, n_tok, &p.k, &nk);
  if (st == UC_OK) st = check_rows(v, fn, "v", batch, n_kv_heads, n_tok, &p.v, &nv);
  if (st == UC_OK) st = check_rows(out, fn, "out", batch, n_q_heads, n_tok, &p.out, &no);
  if (st != UC_OK) return st;
  if (log_decay == nullptr || state_out == nullptr || !aligned(state_out, 16) || !aligned(state_in, 16)) {
    set_error("uc_linear_attend: log_decay and state_out must be non-null, states 16-byte aligned");
    return UC_ERR_ARG;
  }
  const uint64_t ns = 4ull * batch * n_kv_heads * UC_HEAD_DIM * UC_HEAD_DIM;
  if (out->ptr == q->ptr || out->ptr == k->ptr || out->ptr == v->ptr ||
      (state_in != state_out && overlap(state_in, state_in ? ns : 0, state_out, ns))) {
    set_error("uc_linear_attend: outputs overlap inputs");
    return UC_ERR_ARG;
  }
  for (int j = 0; j < n_kv_heads; ++j) {
    if (!std::isfinite(log_decay[j]) || log_decay[j] > 0.f) {
      set_error("uc_linear_attend: log_decay[%d] must be finite and <= 0", j);
      return UC_ERR_ARG;
    }
    const double g = std::exp((double)log_decay[j]), l = (double)log_decay[j] * 1.4426950408889634074;
    p.decay[j] = two_floats(g);
    p.log2_decay[j] = two_floats(std::max(l, -1e30));  // (finite: 0 times it is 0)
  }
  for (int b = 0; b < batch; ++b) {
    p.lengths[b] = lengths ? lengths[b] : n_tok;
    if (p.lengths[b] < 0 || p.lengths[b] > n_tok) {
      set_error("uc_linear_attend: lengths[%d] = %d outside [0, %d]", b, p.lengths[b], n_tok);
      return UC_ERR_SHAPE;
    }
  }
  p.state_in = state_in;
  p.state_out = state_out;
  p.batch = batch;
  p.n_q_heads = n_q_heads;
  p.n_kv_heads = n_kv_heads;
  p.group = n_q_heads / n_kv_heads;
  p.n_tok = n_tok;
  p.scale = (float)(1.0 / std::sqrt((double)UC_HEAD_DIM));
  const cudaStream_t cs = reinterpret_cast<cudaStream_t>(stream);
  // (rows of different tensors may interleave in one buffer)
  auto check_shared = [&]() -> uc_status {
    const RowSet rows[4] = {{&p.out, {batch, n_q_heads, n_tok}, no},
                            {&p.q, {batch, n_q_heads, n_tok}, nq},
                            {&p.k, {batch, n_kv_heads, n_tok}, nk},
                            {&p.v, {batch, n_kv_heads, n_tok}, nv}};
    if (rows_meet(rows[0], rows[0])) {
      set_error("uc_linear_attend: rows of out overlap one another");
      return UC_ERR_SHAPE;
    }
    bool shared = state_in != nullptr && rows_meet(rows[0], state_in, ns);
    for (int i = 0; i < 4; ++i) shared |= (i > 0 && rows_meet(rows[0], rows[i])) || rows_meet(rows[i], state_out, ns);
    if (shared) {
      set_error("uc_linear_attend: outputs overlap inputs or each other");
      return UC_ERR_ARG;
    }
    return UC_OK;
  };
  if (linear_steps(n_q_heads, n_kv_heads, n_tok)) {
    st = check_workspace(workspace, workspace_bytes, 256, "uc_linear_attend");
    if (st == UC_OK) st = check_shared();
    if (st != UC_OK) return st;
    launch_linear_step(p, cs);
    return cuda_check("uc_linear_attend");
  }
  LinearChunkParams c;
  memset(&c, 0, sizeof(c));
  c.plan = plan_linear(batch, n_q_heads, n_kv_heads, p.lengths);
  // (in place, a CTA may write a state that others have yet to start from)
  c.from_start = c.plan.several || (c.plan.head_parts > 1 && state_in == state_out);
  const uint64_t states = c.from_start ? (uint64_t)c.plan.runs * n_kv_heads : 0;
  st = check_workspace(workspace, workspace_bytes, linear_bytes(states), "uc_linear_attend");
  if (st == UC_OK) st = check_shared();
  if (st != UC_OK) return st;
  c.p = p;
  st = encode_rows_4d(&c.tq, p.q, n_tok, n_q_heads, batch, kChunk);
  if (st == UC_OK) st = encode_rows_4d(&c.tk, p.k, n_tok, n_kv_heads, batch, kChunk);
  if (st == UC_OK) st = encode_rows_4d(&c.tv, p.v, n_tok, n_kv_heads, batch, kChunk);
  if (st != UC_OK) return st;
  c.local = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + 256);
  c.start = c.local + states * UC_HEAD_DIM * UC_HEAD_DIM;
  c.status = static_cast<DevStatus*>(workspace);
  c.wait_ns = wait_limit_ns();
  const int withhold = take_withhold_pos();
  c.withhold = c.plan.several ? -1 : withhold;
  c.withhold_sum = c.plan.several ? withhold : -1;
  launch_linear_chunks(c, cs);
  return cuda_check("uc_linear_attend");
}

// --------------------------------------------------------- beam selection
// Vectors of 16 bytes of a row, the first of which may start before it.
static int64_t row_vecs(int32_t vocab, int element) {
  const int per = 16 / element;
  return ((int64_t)vocab + (per - 1) + (per - 1)) / per;
}
static int64_t most_tiles(int64_t vecs) { return vecs < 64 * kBeamMinSpan ? (vecs + kBeamMinSpan - 1) / kBeamMinSpan : 64; }
// Vectors per tile: the split of the rows that the SMs are through with first.
// kStart is a CTA's start, first bound and ranking, in vectors' time. Compared over
// 1 to 512 rows of 32000, 65537 and 150001 logits in bf16 and fp32 (60 shapes, one
// to eight beams): with 2048 each is within 6 % of the best of all; with 512 or
// 1024 long rows are cut too often (256 rows of 150001: 40 us instead of 30 in
// bf16, 50 instead of 38 in fp32), with 4096 or 8192 others too seldom (160 rows
// of 65537: 19 instead of 17), with none each takes up to five times as long.
static int beam_span(int64_t rows, int n_beams, int64_t vecs, int64_t slots) {
  constexpr int64_t kStart = 2048;
  int64_t best = vecs, cost = INT64_MAX;
  for (int64_t t = 1; t <= most_tiles(vecs) && t * n_beams <= kBeamLists; ++t) {
    const int64_t span = ((vecs + t - 1) / t + 31) / 32 * 32;
    const int64_t c = (rows * t + slots - 1) / slots * (kStart + span);
    if (c < cost) {
      cost = c;
      best = span;
    }
  }
  return (int)best;
}

size_t uc_beam_workspace_size(int32_t batch, int32_t n_beams, int32_t vocab, int32_t n) {
  UC_TRACE();
  if (batch < 1 || n_beams < 1 || vocab < 1 || n < 1) return 0;
  const uint64_t lists = (uint64_t)batch * n_beams * most_tiles(row_vecs(vocab, 4));  // (the most of any type)
  return 256 + lists * (sizeof(float2) + (uint64_t)n * 8);
}

uc_status uc_beam_select(const void* logits, int32_t dtype, int64_t stride_b, int64_t stride_k, int32_t batch,
                         int32_t n_beams, int32_t vocab, const float* scores, const uint8_t* finished, int32_t eos,
                         int32_t n, float* out_scores, int32_t* out_parent, int32_t* out_token,
                         uint8_t* out_finished, void* workspace, size_t workspace_bytes, void* stream) {
  UC_TRACE();
  if (dtype != UC_FP32 && dtype != UC_BF16 && dtype != UC_FP16) {
    set_error("uc_beam_select: bad logits type %d", dtype);
    return UC_ERR_ARG;
  }
  if (batch < 1 || n_beams < 1 || n_beams > UC_MAX_BEAMS || vocab < 1 || n < 1 || n > UC_MAX_BEAM_OUT ||
      (int64_t)batch * n_beams > 65535 || n > (int64_t)n_beams * vocab) {
    set_error("uc_beam_select: unsupported shape (batch %d, beams %d, vocabulary %d, n %d)", batch, n_beams, vocab, n);
    return UC_ERR_SHAPE;
  }
  if ((n_beams > 1 && stride_k < vocab) || (batch > 1 && stride_b < 1)) {
    set_error("uc_beam_select: logits rows overlap (strides %lld, %lld)", (long long)stride_b, (long long)stride_k);
    return UC_ERR_SHAPE;
  }
  if (logits == nullptr || scores == nullptr || out_scores == nullptr || out_parent == nullptr ||
      out_token == nullptr || !aligned(logits, dtype == UC_FP32 ? 4 : 2) || !aligned(scores, 4) ||
      !aligned(out_scores, 4) || !aligned(out_parent, 4) || !aligned(out_token, 4)) {
    set_error("uc_beam_select: null or misaligned argument");
    return UC_ERR_ARG;
  }
  if (eos < -1 || eos >= vocab || (finished != nullptr && eos < 0)) {
    set_error("uc_beam_select: end token %d outside the vocabulary (%d), or finished beams without one", eos, vocab);
    return UC_ERR_ARG;
  }
  const uc_status st = check_workspace(workspace, workspace_bytes, uc_beam_workspace_size(batch, n_beams, vocab, n),
                                       "uc_beam_select");
  if (st != UC_OK) return st;
  // (a request's scores are read before its results are written, so they may take their place)
  struct { const void* p; uint64_t bytes; } out[4] = {{out_scores, 4ull * batch * n}, {out_parent, 4ull * batch * n},
                                                      {out_token, 4ull * batch * n},
                                                      {out_finished, out_finished ? 1ull * batch * n : 0}};
  for (int i = 0; i < 4; ++i) {
    bool shared = overlap(out[i].p, out[i].bytes, finished, finished ? 1ull * batch * n_beams : 0) ||
                  (!(i == 0 && out_scores == scores && n == n_beams) &&
                   overlap(out[i].p, out[i].bytes, scores, 4ull * batch * n_beams));
    for (int j = 0; j < i; ++j) shared |= overlap(out[i].p, out[i].bytes, out[j].p, out[j].bytes);
    if (shared) {
      set_error("uc_beam_select: outputs overlap inputs or each other");
      return UC_ERR_ARG;
    }
  }
  BeamParams p;
  memset(&p, 0, sizeof(p));
  p.logits = logits;
  p.stride_b = batch > 1 ? stride_b : 0;
  p.stride_k = n_beams > 1 ? stride_k : 0;
  p.scores = scores;
  p.finished = finished;
  p.out_scores = out_scores;
  p.out_parent = out_parent;
  p.out_token = out_token;
  p.out_finished = out_finished;
  p.batch = batch;
  p.beams = n_beams;
  p.vocab = vocab;
  p.n = n;
  const int64_t vecs = row_vecs(vocab, dtype == UC_FP32 ? 4 : 2);
  p.span = beam_span((int64_t)batch * n_beams, n_beams, vecs, kBeamPerSm * num_sms());
  p.tiles = (int)((vecs + p.span - 1) / p.span);
  p.eos = eos;
  p.status = static_cast<DevStatus*>(workspace);
  const size_t lists = (size_t)batch * n_beams * p.tiles;
  p.part_ms = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + 256);
  p.part_x = reinterpret_cast<float*>(p.part_ms + lists);
  p.part_tok = reinterpret_cast<int32_t*>(p.part_x + lists * n);
  launch_beam(p, dtype, reinterpret_cast<cudaStream_t>(stream));
  return cuda_check("uc_beam_select");
}

// ---------------------------------------------------------------- reorder
namespace {

struct ReorderList {
  ReorderParams p;
  cudaStream_t stream;
  int64_t units = 0;
  bool launched = false;

  void flush() {
    if (p.n_arrays == 0) return;
    p.n_units = (int32_t)units;
    launch_reorder(p, stream);
    p.n_arrays = 0;
    units = 0;
  }
  void add(const void* src, void* dst, int64_t src_block, int64_t dst_block, int heads, int unit, int live,
           int max_units, const int32_t* n_kept, int max_kept) {
    const int64_t parts = ((int64_t)max_units * unit + kReorderBytes - 1) / kReorderBytes;
    const int64_t more = parts * heads * p.n_seq;
    if (more == 0) return;
    if (p.n_arrays == kReorderArrays || units + more > INT32_MAX) flush();
    ReorderArray& a = p.a[p.n_arrays++];
    a.src = static_cast<const uint8_t*>(src);
    a.dst = static_cast<uint8_t*>(dst);
    a.src_block = src_block;
    a.dst_block = dst_block;
    a.n_kept = n_kept;
    a.heads = heads;
    a.unit = unit;
    a.live = live;
    a.max_units = max_units;
    a.max_kept = max_kept;
    a.parts = (int32_t)parts;
    a.begin = (int32_t)units;
    units += more;
  }
};

bool packed(const uc_segment* s) { return s->kind == UC_KIND_QUANT || s->kind == UC_KIND_EVICT_QUANT; }

// Tokens a block of the segment can hold.
int capacity(const uc_segment* s) { return s->kind == UC_KIND_FULL ? s->n_src : s->cap; }

uc_status check_item(const uc_reorder_item& it, int i, int n_groups, int n_from, int n_to) {
  if ((it.src == nullptr) != (it.dst == nullptr) || (it.state_src == nullptr) != (it.state_dst == nullptr) ||
      (it.src == nullptr) == (it.state_src == nullptr)) {
    set_error("uc_reorder: item %d is neither a pair of segments nor a pair of arrays", i);
    return UC_ERR_ARG;
  }
  if (it.src == nullptr) {
    if (it.state_bytes == 0 || it.state_bytes % 4 != 0 || it.state_bytes > INT32_MAX || !aligned(it.state_src, 4) ||
        !aligned(it.state_dst, 4)) {
      set_error("uc_reorder: item %d: %llu bytes per sequence (a multiple of 4 below 2^31, 4-byte aligned arrays)", i,
                (unsigned long long)it.state_bytes);
      return UC_ERR_SHAPE;
    }
    if (overlap(it.state_src, it.state_bytes * n_groups * n_from, it.state_dst, it.state_bytes * n_groups * n_to)) {
      set_error("uc_reorder: item %d: source and target overlap", i);
      return UC_ERR_ARG;
    }
    return UC_OK;
  }
  const uc_segment *s = it.src, *d = it.dst;
  uc_status st = check_segment(s, "uc_reorder");
  if (st == UC_OK) st = check_segment(d, "uc_reorder");
  if (st != UC_OK) return st;
  if (s->kind != d->kind || s->bits != d->bits || s->n_kv_heads != d->n_kv_heads || s->n_src != d->n_src ||
      capacity(d) < capacity(s) || s->batch != n_groups * n_from || d->batch != n_groups * n_to) {
    set_error("uc_reorder: item %d: segments differ (kind, bits, heads or source length), the target is smaller, or "
              "their batches are not %d x %d and %d x %d", i, n_groups, n_from, n_groups, n_to);
    return UC_ERR_SHAPE;
  }
  for (int g = 0; g < n_groups; ++g)
    for (int j = 1; j < n_from; ++j)
      if (s->n_kept_host[g * n_from + j] != s->n_kept_host[g * n_from]) {
        set_error("uc_reorder: item %d: the sequences of group %d hold different numbers of tokens", i, g);
        return UC_ERR_SHAPE;
      }
  for (const uc_segment* x : {s, d}) {
    const int64_t last = ((int64_t)x->batch * x->n_kv_heads - 1) * x->row_stride + x->row_offset +
                         (packed(x) ? UC_GROUP : capacity(x));
    if (last > x->rows_total || x->row_stride < (packed(x) ? UC_GROUP : capacity(x))) {
      set_error("uc_reorder: item %d: rows run past rows_total, or blocks overlap", i);
      return UC_ERR_SHAPE;
    }
  }
  uc_segment_sizes zs, zd;
  st = uc_segment_sizes_of(s, &zs);
  if (st == UC_OK) st = uc_segment_sizes_of(d, &zd);
  if (st != UC_OK) return st;
  const uint64_t ns = (uint64_t)s->rows_total * UC_HEAD_DIM * 2, nd = (uint64_t)d->rows_total * UC_HEAD_DIM * 2;
  if (overlap(s->k, ns, d->k, nd) || overlap(s->v, ns, d->v, nd) || overlap(s->n_kept, zs.n_kept, d->n_kept, zd.n_kept) ||
      overlap(s->kept_idx, zs.kept_idx, d->kept_idx, zd.kept_idx) ||
      overlap(s->k_codes, zs.k_codes, d->k_codes, zd.k_codes) ||
      overlap(s->v_codes, zs.v_codes, d->v_codes, zd.v_codes) ||
      overlap(s->k_params, zs.k_params, d->k_params, zd.k_params) ||
      overlap(s->v_params, zs.v_params, d->v_params, zd.v_params)) {
    set_error("uc_reorder: item %d: source and target share storage", i);
    return UC_ERR_ARG;
  }
  return UC_OK;
}

}  // namespace

uc_status uc_reorder(const uc_reorder_item* items, int32_t n_items, const int32_t* parent, int32_t n_groups,
                     int32_t n_from, int32_t n_to, void* workspace, size_t workspace_bytes, void* stream) {
  UC_TRACE();
  if (items == nullptr || parent == nullptr || !aligned(parent, 4)) {
    set_error("uc_reorder: null or misaligned argument");
    return UC_ERR_ARG;
  }
  if (n_items < 1 || n_groups < 1 || n_from < 1 || n_to < 1 || (int64_t)n_groups * n_from > 65535 ||
      (int64_t)n_groups * n_to > 65535) {
    set_error("uc_reorder: bad sizes (%d items, %d groups, %d -> %d)", n_items, n_groups, n_from, n_to);
    return UC_ERR_SHAPE;
  }
  uc_status st = check_workspace(workspace, workspace_bytes, 256, "uc_reorder");
  if (st != UC_OK) return st;
  for (int i = 0; i < n_items; ++i) {
    st = check_item(items[i], i, n_groups, n_from, n_to);
    if (st != UC_OK) return st;
  }
  ReorderList list;
  list.stream = reinterpret_cast<cudaStream_t>(stream);
  list.p.parent = parent;
  list.p.status = static_cast<DevStatus*>(workspace);
  list.p.n_arrays = 0;
  list.p.n_seq = n_groups * n_to;
  list.p.n_from = n_from;
  list.p.n_to = n_to;
  for (int i = 0; i < n_items; ++i) {
    const uc_reorder_item& it = items[i];
    if (it.src == nullptr) {
      const int bytes = (int)it.state_bytes;
      list.add(it.state_src, it.state_dst, bytes, bytes, 1, 4, kLiveAll, bytes / 4, nullptr, 0);
      continue;
    }
    const uc_segment* s = it.src;
    uc_segment* d = it.dst;
    const int h = s->n_kv_heads, cap = capacity(s);
    constexpr int kRow = UC_HEAD_DIM * 2;
    const int64_t so = s->row_offset * kRow, dof = d->row_offset * kRow;
    const int64_t sb = s->row_stride * kRow, db = d->row_stride * kRow;
    auto shifted = [](void* p, int64_t off) { return static_cast<void*>(static_cast<uint8_t*>(p) + off); };
    if (packed(s)) {
      const int codes = UC_GROUP * UC_HEAD_DIM * s->bits / 8, groups = cap / UC_GROUP;
      const int64_t sg = s->cap / UC_GROUP, dg = d->cap / UC_GROUP;
      list.add(s->k_codes, d->k_codes, sg * codes, dg * codes, h, codes, kLiveGroups, groups, s->n_kept, cap);
      list.add(s->v_codes, d->v_codes, sg * codes, dg * codes, h, codes, kLiveGroups, groups, s->n_kept, cap);
      list.add(s->k_params, d->k_params, sg * 512, dg * 512, h, 512, kLiveGroups, groups, s->n_kept, cap);
      list.add(s->v_params, d->v_params, sg * 512, dg * 512, h, 512, kLiveGroups, groups, s->n_kept, cap);
      list.add(s->k, d->k, sb, db, h, kRow, kLiveTail, UC_GROUP - 1, s->n_kept, cap);
      list.add(s->v, d->v, sb, db, h, kRow, kLiveTail, UC_GROUP - 1, s->n_kept, cap);
    } else {
      list.add(shifted(s->k, so), shifted(d->k, dof), sb, db, h, kRow, kLiveTokens, cap, s->n_kept, cap);
      list.add(shifted(s->v, so), shifted(d->v, dof), sb, db, h, kRow, kLiveTokens, cap, s->n_kept, cap);
    }
    if (s->kind != UC_KIND_FULL)
      list.add(s->kept_idx, d->kept_idx, 4ll * s->cap, 4ll * d->cap, h, 4, kLiveTokens, cap, s->n_kept, cap);
    list.add(s->n_kept, d->n_kept, 4, 4, 1, 4, kLiveCount, 1, s->n_kept, cap);
  }
  list.flush();
  st = cuda_check("uc_reorder");
  if (st == UC_OK)
    for (int i = 0; i < n_items; ++i)
      if (items[i].src != nullptr)
        for (int j = 0; j < n_groups * n_to; ++j)
          items[i].dst->n_kept_host[j] = items[i].src->n_kept_host[j / n_to * n_from];
  return st;
}

}  // extern "C"
