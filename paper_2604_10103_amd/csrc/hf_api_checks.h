// Checks of the arguments of rotations, norms and the caches of pages, shared by their entry points (internal, host only).
#pragma once

#include <math.h>

#include <numeric>

#include "hf_common.h"

namespace hf {

#define HF_TRY(expr) do { int _r = (expr); if (_r != HF_OK) return _r; } while (0)


inline int check_ptr(const void* p, const char* name, unsigned align = 16) {
  if (!p) { set_error("%s is NULL", name); return HF_ERR_NULL; }
  if (reinterpret_cast<uintptr_t>(p) & (align - 1)) { set_error("%s is not %u-byte aligned", name, align); return HF_ERR_ALIGN; }
  return HF_OK;
}

inline int check_rows(int32_t n, const char* name) {
  if (n < 0 || n > (1 << 24)) { set_error("%s must be in [0, 2^24], got %d", name, n); return HF_ERR_SHAPE; }
  return HF_OK;
}

inline int check_type(int32_t dtype, int32_t head_dim) {
  if (head_dim != 64 && head_dim != 128) { set_error("head_dim must be 64 or 128, got %d", head_dim); return HF_ERR_SHAPE; }
  if (dtype != HF_BF16 && dtype != HF_F32) { set_error("unknown dtype %d", dtype); return HF_ERR_DTYPE; }
  return HF_OK;
}

inline int check_rope(const hf_rope_axes* r, int head_dim) {
  if (!r) { set_error("rope is NULL"); return HF_ERR_NULL; }
  if (r->n_axes < 1 || r->n_axes > HF_ROPE_MAX_AXES) { set_error("n_axes must be in [1, %d], got %d", HF_ROPE_MAX_AXES, r->n_axes); return HF_ERR_SHAPE; }
  int pairs = 0;
  for (int a = 0; a < r->n_axes; ++a) {
    if (r->pairs[a] < 1 || r->pairs[a] > head_dim / 2 - pairs) {
      set_error("pairs must be >= 1 each and at most head_dim / 2 = %d together", head_dim / 2);
      return HF_ERR_SHAPE;
    }
    pairs += r->pairs[a];
  }
  if (!(r->theta >= 1.0) || !isfinite(r->theta)) { set_error("theta must be finite and >= 1"); return HF_ERR_SHAPE; }
  if (r->layout != HF_ROPE_ADJACENT && r->layout != HF_ROPE_HALVES) { set_error("unknown layout %d", r->layout); return HF_ERR_DTYPE; }
  if (r->spectrum != HF_ROPE_PER_AXIS && r->spectrum != HF_ROPE_SHARED) { set_error("unknown spectrum %d", r->spectrum); return HF_ERR_DTYPE; }
  return HF_OK;
}

inline int check_cache(const hf_paged* c) {
  if (!c) { set_error("cache is NULL"); return HF_ERR_NULL; }
  HF_TRY(check_type(c->dtype, c->head_dim));
  if (c->heads < 1 || c->heads > 65535 || c->heads_kv < 1 || c->heads % c->heads_kv != 0) {
    set_error("heads must be in [1, 65535] and a multiple of heads_kv, got %d and %d", c->heads, c->heads_kv);
    return HF_ERR_SHAPE;
  }
  if (c->page_tokens < 1 || c->page_tokens > 65536) { set_error("page_tokens must be in [1, 65536], got %d", c->page_tokens); return HF_ERR_SHAPE; }
  if (c->n_pages < 1) { set_error("n_pages must be >= 1"); return HF_ERR_SHAPE; }
  if (c->n_seqs < 1 || c->n_seqs > 65535) { set_error("n_seqs must be in [1, 65535], got %d", c->n_seqs); return HF_ERR_SHAPE; }
  if (c->max_pages < 1 || (int64_t)c->max_pages * c->page_tokens > (1 << 30)) {
    set_error("max_pages must be >= 1 and max_pages * page_tokens <= 2^30");
    return HF_ERR_SHAPE;
  }
  if (c->window < 0 || c->n_sink < 0) { set_error("window and n_sink must be >= 0"); return HF_ERR_SHAPE; }
  if (!(c->softmax_scale >= 0.0f) || !isfinite(c->softmax_scale)) { set_error("softmax_scale is invalid"); return HF_ERR_SHAPE; }
  return HF_OK;
}

// A strided operand of up to three outer dimensions (outermost first) and rows of `row` elements
struct View {
  const char* p;
  int64_t n[3], stride[3], row;
  int dims, es;
  // bytes from p to behind the last element
  int64_t span() const {
    int64_t last = 0;
    for (int i = 0; i < dims; ++i) last += (n[i] - 1) * stride[i];
    return (last + row) * es;
  }
};

inline int check_view(View& v, const void* p, const char* name, const int64_t* strides, const int64_t* defaults, bool written) {
  HF_TRY(check_ptr(p, name));
  v.p = static_cast<const char*>(p);
  for (int i = 0; i < v.dims; ++i) {
    v.stride[i] = strides ? strides[i] : defaults[i];
    if (v.stride[i] < 0 || v.stride[i] > (1ll << 36)) { set_error("a stride of %s is outside [0, 2^36]", name); return HF_ERR_SHAPE; }
    if (v.n[i] > 1 && v.stride[i] * v.es % 16 != 0) { set_error("a stride of %s is no multiple of 16 bytes", name); return HF_ERR_ALIGN; }
  }
  if (written) {   // every stride covers what the smaller ones span
    int64_t covered = v.row;
    bool done[3] = {false, false, false};
    for (int k = 0; k < v.dims; ++k) {
      int at = -1;
      for (int i = 0; i < v.dims; ++i)
        if (!done[i] && v.n[i] > 1 && (at < 0 || v.stride[i] < v.stride[at])) at = i;
      if (at < 0) break;
      done[at] = true;
      if (v.stride[at] < covered) { set_error("rows of %s overlap each other", name); return HF_ERR_SHAPE; }
      covered = v.stride[at] * (v.n[at] - 1) + covered;
    }
  }
  return HF_OK;
}

// in place, or apart
inline int check_apart(const View& x, const View& y, const char* what, bool in_place) {
  if (in_place && x.p == y.p) {
    bool same = true;
    for (int i = 0; i < x.dims; ++i) same = same && (x.n[i] <= 1 || x.stride[i] == y.stride[i]);
    if (same) return HF_OK;
  }
  if (x.p < y.p + y.span() && y.p < x.p + x.span()) { set_error("%s", what); return HF_ERR_SHAPE; }
  return HF_OK;
}

inline bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  const char *x = static_cast<const char*>(a), *y = static_cast<const char*>(b);
  return x < y + nb && y < x + na;
}

// Whether x and y can be shown to have no byte in common though their rows may interleave (rows of one joint projection): for some period T,
// what x covers of the places modulo T, an interval that its strides which T divides do not widen, lies beside what y covers.  Candidates are
// their strides and the strides' common divisors
inline bool interleave(const View& x, const View& y) {
  if (!overlap(x.p, x.span(), y.p, y.span())) return true;
  const auto beside = [&](int64_t T) {
    const auto width = [&](const View& v) {
      int64_t w = v.row * v.es;
      for (int i = 0; i < v.dims; ++i)
        if (v.stride[i] * v.es % T != 0) w += (v.n[i] - 1) * v.stride[i] * v.es;
      return w;
    };
    const int64_t wx = width(x), wy = width(y), d = ((y.p - x.p) % T + T) % T;   // (x at 0, y at d)
    return d >= wx && d + wy <= T;
  };
  const auto period = [](const View& v, int i) { return v.n[i] > 1 ? v.stride[i] * v.es : 0; };
  for (int i = 0; i < x.dims; ++i)
    if (period(x, i) > 0 && beside(period(x, i))) return true;
  for (int j = 0; j < y.dims; ++j) {
    if (period(y, j) > 0 && beside(period(y, j))) return true;
    for (int i = 0; i < x.dims; ++i)
      if (period(x, i) > 0 && period(y, j) > 0 && beside(std::gcd(period(x, i), period(y, j)))) return true;
  }
  return false;
}

// queries that are written while other workgroups read the new keys and values
inline int check_queries_apart(const View& q_out, const View& k, const View& v) {
  for (const View* x : {&k, &v})
    if (!interleave(q_out, *x)) { set_error("Q_out overlaps %s", x == &k ? "K_new" : "V_new"); return HF_ERR_SHAPE; }
  return HF_OK;
}

// What the call writes must not lie over what its later workgroups read
inline int check_reads(const void* written, int64_t bytes, const char* name, const hf_paged& c, const int32_t* cu_new, const int32_t* seq_lens,
                const int32_t* page_table, const int32_t* positions = nullptr, int64_t n_positions = 0) {
  const struct { const int32_t* p; int64_t n; const char* name; } reads[] = {{cu_new, (int64_t)c.n_seqs + 1, "cu_new"},
                                                                             {seq_lens, c.n_seqs, "seq_lens"},
                                                                             {page_table, (int64_t)c.n_seqs * c.max_pages, "page_table"},
                                                                             {positions, n_positions, "positions"}};
  for (const auto& r : reads)
    if (r.p && overlap(written, bytes, r.p, 4 * r.n)) { set_error("%s overlaps %s", name, r.name); return HF_ERR_SHAPE; }
  return HF_OK;
}

inline int64_t pool_bytes(const hf_paged& c) {
  return (int64_t)c.n_pages * c.heads_kv * c.page_tokens * c.head_dim * (c.dtype == HF_BF16 ? 2 : 4);
}

inline int check_pool(const hf_paged* c, const void* K_pages, const void* V_pages, const int32_t* page_table, const int32_t* cu_new, const int32_t* seq_lens) {
  HF_TRY(check_ptr(cu_new, "cu_new", 4));
  HF_TRY(check_ptr(seq_lens, "seq_lens", 4));
  HF_TRY(check_ptr(K_pages, "K_pages"));
  HF_TRY(check_ptr(V_pages, "V_pages"));
  HF_TRY(check_ptr(page_table, "page_table", 4));
  // (rows of the pool count in 32 bits: 512 GB at least)
  if ((unsigned __int128)c->n_pages * c->heads_kv * c->page_tokens >= ((unsigned __int128)1 << 32)) {
    set_error("n_pages * heads_kv * page_tokens must be < 2^32");
    return HF_ERR_SHAPE;
  }
  return HF_OK;
}

inline View packed(const hf_paged& c, int n, int heads) {
  View v = {};
  v.dims = 2;
  v.n[0] = n;
  v.n[1] = heads;
  v.row = c.head_dim;
  v.es = c.dtype == HF_BF16 ? 2 : 4;
  return v;
}

inline int check_packed(View& v, const void* p, const char* name, const int64_t* strides, bool written) {
  const int64_t defaults[2] = {v.n[1] * v.row, v.row};
  return check_view(v, p, name, strides, defaults, written);
}

}  // namespace hf
