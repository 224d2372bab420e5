// Argument checks shared by the C-ABI entry points over rows of any strides:
// alignment, overlap, workspaces. Host code only.
#pragma once

#include <algorithm>

#include "internal.h"

namespace uc {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Do [a, a + an) and [b, b + bn) share a byte?
inline bool overlap(const void* a, uint64_t an, const void* b, uint64_t bn) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return an != 0 && bn != 0 && x < y + bn && y < x + an;
}

inline uc_status check_workspace(const void* workspace, size_t bytes, size_t need, const char* fn) {
  if (workspace == nullptr || !aligned(workspace, 16)) {
    set_error("%s: workspace must be non-null and 16-byte aligned", fn);
    return UC_ERR_ARG;
  }
  if (bytes < need) {
    set_error("%s: workspace of %zu bytes, %zu needed", fn, bytes, need);
    return UC_ERR_OOM;
  }
  return UC_OK;
}

constexpr int64_t kMostElements = int64_t(1) << 44;  // between two rows of one tensor

// stride * x, lo <= x <= hi.
struct Term {
  int64_t stride, lo, hi;
};

// Is there a sum d + stride_0 x_0 + ... strictly between -before and after (all x
// zero: only if `zero`)? Terms by falling stride: what the later ones reach
// leaves few x to look at, one or two each where strides nest. A search that
// grows past `steps` counts as found.
inline bool reaches(const Term* t, int n, int64_t d, int64_t before, int64_t after, bool zero, int* steps) {
  if (n == 0) return zero && d > -before && d < after;
  int64_t lo = 0, hi = 0;
  for (int i = 1; i < n; ++i) {
    lo += t[i].stride * t[i].lo;
    hi += t[i].stride * t[i].hi;
  }
  auto floor_div = [](int64_t a, int64_t b) { return a / b - (a % b < 0); };
  const int64_t first = std::max(t->lo, floor_div(-before - d - hi, t->stride) + 1);
  const int64_t last = std::min(t->hi, -floor_div(-(after - d - lo), t->stride) - 1);
  for (int64_t x = first; x <= last; ++x)
    if (--*steps < 0 || reaches(t + 1, n - 1, d + t->stride * x, before, after, zero || x != 0, steps)) return true;
  return false;
}

// Rows of a tensor: [batch, heads, tokens] of UC_HEAD_DIM elements.
struct RowSet {
  const RowsDev* r;
  int size[3];
  uint64_t bytes;   // from the first row to the last's end
  int element = 2;  // bytes of one
  int64_t stride(int i) const { return i == 0 ? r->sb : i == 1 ? r->sh : r->st; }
};

// Does a row of a share an element with a row of b, of the same type (with another row, where both are one)?
inline bool rows_meet(const RowSet& a, const RowSet& b) {
  const bool same = &a == &b;
  if (!same && !overlap(a.r->base, a.bytes, b.r->base, b.bytes)) return false;
  Term t[6];
  int n = 0;
  for (int i = 0; i < 3; ++i) {
    if (a.size[i] > 1 && b.size[i] > 1 && a.stride(i) == b.stride(i)) {
      t[n++] = {a.stride(i), 1 - b.size[i], a.size[i] - 1};
    } else {
      if (a.size[i] > 1) t[n++] = {a.stride(i), 0, a.size[i] - 1};
      if (b.size[i] > 1) t[n++] = {b.stride(i), 1 - b.size[i], 0};
    }
  }
  std::sort(t, t + n, [](const Term& x, const Term& y) { return x.stride > y.stride; });
  int steps = 1 << 16;
  const int64_t d = ((int64_t)reinterpret_cast<uintptr_t>(a.r->base) - (int64_t)reinterpret_cast<uintptr_t>(b.r->base)) / a.element;
  return reaches(t, n, d, UC_HEAD_DIM, UC_HEAD_DIM, !same, &steps);
}

// Does a row of a share a byte with the `bytes` bytes at x?
inline bool rows_meet(const RowSet& a, const void* x, uint64_t bytes) {
  if (!overlap(a.r->base, a.bytes, x, bytes)) return false;
  Term t[3];
  int n = 0;
  for (int i = 0; i < 3; ++i)
    if (a.size[i] > 1) t[n++] = {a.stride(i), 0, a.size[i] - 1};
  std::sort(t, t + n, [](const Term& x, const Term& y) { return x.stride > y.stride; });
  int steps = 1 << 16;
  const int64_t d = ((int64_t)reinterpret_cast<uintptr_t>(a.r->base) - (int64_t)reinterpret_cast<uintptr_t>(x)) / a.element;
  return reaches(t, n, d, UC_HEAD_DIM, (int64_t)(bytes / a.element), true, &steps);
}

// Rows of `heads` heads of `n_tok` tokens: strides in the kernels' form (0
// where the extent is 1) and the bytes from the first row to the last's end.
inline uc_status check_rows(const uc_rows* r, const char* fn, const char* what, int batch, int heads, int n_tok,
                            RowsDev* out, uint64_t* extent, int element = 2) {
  if (r == nullptr || r->ptr == nullptr || !aligned(r->ptr, 16)) {
    set_error("%s: %s must be non-null and 16-byte aligned", fn, what);
    return UC_ERR_ARG;
  }
  const int64_t stride[3] = {batch > 1 ? r->stride_b : 0, heads > 1 ? r->stride_h : 0, n_tok > 1 ? r->stride_t : 0};
  const int size[3] = {batch, heads, n_tok};
  int64_t last = 0;
  for (int i = 0; i < 3; ++i) {
    if (size[i] > 1 && (stride[i] < UC_HEAD_DIM || stride[i] % 8 != 0 || stride[i] > (int64_t(1) << 37))) {
      set_error("%s: strides of %s must be multiples of 8 elements, at least %d and below 2^37", fn, what, UC_HEAD_DIM);
      return UC_ERR_SHAPE;
    }
    if (size[i] > 1 && stride[i] > kMostElements / (size[i] - 1)) {
      set_error("%s: rows of %s lie more than 2^44 elements apart", fn, what);
      return UC_ERR_SHAPE;
    }
    last += stride[i] * (size[i] - 1);
  }
  *out = RowsDev{static_cast<__nv_bfloat16*>(r->ptr), stride[0], stride[1], stride[2]};
  *extent = (uint64_t)element * (uint64_t)(last + UC_HEAD_DIM);
  return UC_OK;
}

// The rows of a window's cache, in the kernels' form.
inline uc_status check_window_cache(const uc_window_cache* c, const char* fn, RowsDev* k, RowsDev* v, uint64_t* nk,
                                    uint64_t* nv) {
  if (c == nullptr) {
    set_error("%s: no cache", fn);
    return UC_ERR_ARG;
  }
  if (c->batch < 1 || c->batch > 65535 || c->n_kv_heads < 1 || c->n_kv_heads > 65535 || c->n_rows < 1 ||
      c->n_rows > (1 << 30) || c->window < 1 || c->n_sink < 0) {
    set_error("%s: unsupported cache (batch %d, kv heads %d, %d rows, window %d, %d first tokens)", fn, c->batch,
              c->n_kv_heads, c->n_rows, c->window, c->n_sink);
    return UC_ERR_SHAPE;
  }
  uc_status st = check_rows(&c->k, fn, "the cache's k", c->batch, c->n_kv_heads, c->n_rows, k, nk);
  if (st == UC_OK) st = check_rows(&c->v, fn, "the cache's v", c->batch, c->n_kv_heads, c->n_rows, v, nv);
  return st;
}

// n_sink below n_rows, as the kernels need it: of sequences that the rows hold, the last
// row's token is then seen by its own query alone, which has it in its window.
inline uc_window_cache within_rows(const uc_window_cache& c) {
  uc_window_cache r = c;
  r.n_sink = std::min(c.n_sink, c.n_rows - 1);
  return r;
}

}  // namespace uc
