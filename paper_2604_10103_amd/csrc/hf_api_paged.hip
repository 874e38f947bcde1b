// Entry points of the rotation by positions and of the cache of pages: host-side argument checks, then the launch.
#include <math.h>

#include "hf_paged.h"

using namespace hf;

namespace {

#define HF_TRY(expr) do { int _r = (expr); if (_r != HF_OK) return _r; } while (0)

int check_ptr(const void* p, const char* name, unsigned align = 16) {
  if (!p) { set_error("%s is NULL", name); return HF_ERR_NULL; }
  if (reinterpret_cast<uintptr_t>(p) & (align - 1)) { set_error("%s is not %u-byte aligned", name, align); return HF_ERR_ALIGN; }
  return HF_OK;
}

int check_rows(int32_t n, const char* name) {
  if (n < 0 || n > (1 << 24)) { set_error("%s must be in [0, 2^24], got %d", name, n); return HF_ERR_SHAPE; }
  return HF_OK;
}

int check_type(int32_t dtype, int32_t head_dim) {
  if (head_dim != 64 && head_dim != 128) { set_error("head_dim must be 64 or 128, got %d", head_dim); return HF_ERR_SHAPE; }
  if (dtype != HF_BF16 && dtype != HF_F32) { set_error("unknown dtype %d", dtype); return HF_ERR_DTYPE; }
  return HF_OK;
}

int check_rope(const hf_rope_axes* r, int head_dim) {
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

int check_cache(const hf_paged* c) {
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

int check_attn_rows(const hf_paged* c, int32_t n_q) {
  HF_TRY(check_rows(n_q, "n_q"));
  if ((int64_t)n_q * c->heads > (1ll << 30)) { set_error("n_q * heads must be <= 2^30"); return HF_ERR_SHAPE; }
  if (n_q > 0 && paged_threads(*c, n_q) >= (1ll << 32)) { set_error("more rows and sequences than a launch of 2^32 threads holds"); return HF_ERR_SHAPE; }
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

int check_view(View& v, const void* p, const char* name, const int64_t* strides, const int64_t* defaults, bool written) {
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
int check_apart(const View& x, const View& y, const char* what, bool in_place) {
  if (in_place && x.p == y.p) {
    bool same = true;
    for (int i = 0; i < x.dims; ++i) same = same && (x.n[i] <= 1 || x.stride[i] == y.stride[i]);
    if (same) return HF_OK;
  }
  if (x.p < y.p + y.span() && y.p < x.p + x.span()) { set_error("%s", what); return HF_ERR_SHAPE; }
  return HF_OK;
}

bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  const char *x = static_cast<const char*>(a), *y = static_cast<const char*>(b);
  return x < y + nb && y < x + na;
}

// What the call writes must not lie over what its later workgroups read
int check_reads(const void* written, int64_t bytes, const char* name, const hf_paged& c, const int32_t* cu_new, const int32_t* seq_lens,
                const int32_t* page_table, const int32_t* positions = nullptr, int64_t n_positions = 0) {
  const struct { const int32_t* p; int64_t n; const char* name; } reads[] = {{cu_new, (int64_t)c.n_seqs + 1, "cu_new"},
                                                                             {seq_lens, c.n_seqs, "seq_lens"},
                                                                             {page_table, (int64_t)c.n_seqs * c.max_pages, "page_table"},
                                                                             {positions, n_positions, "positions"}};
  for (const auto& r : reads)
    if (r.p && overlap(written, bytes, r.p, 4 * r.n)) { set_error("%s overlaps %s", name, r.name); return HF_ERR_SHAPE; }
  return HF_OK;
}

int64_t pool_bytes(const hf_paged& c) {
  return (int64_t)c.n_pages * c.heads_kv * c.page_tokens * c.head_dim * (c.dtype == HF_BF16 ? 2 : 4);
}

int check_pool(const hf_paged* c, const void* K_pages, const void* V_pages, const int32_t* page_table, const int32_t* cu_new, const int32_t* seq_lens) {
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

View packed(const hf_paged& c, int n, int heads) {
  View v = {};
  v.dims = 2;
  v.n[0] = n;
  v.n[1] = heads;
  v.row = c.head_dim;
  v.es = c.dtype == HF_BF16 ? 2 : 4;
  return v;
}

int check_packed(View& v, const void* p, const char* name, const int64_t* strides, bool written) {
  const int64_t defaults[2] = {v.n[1] * v.row, v.row};
  return check_view(v, p, name, strides, defaults, written);
}

}  // namespace

extern "C" {

int hf_rope_axes_apply(const hf_rope_axes* rope, int32_t dtype, int32_t head_dim, int32_t batch, int32_t heads, int32_t n_tokens,
                       const void* X, const int64_t* x_strides, const int32_t* positions, int32_t positions_per_batch, void* Y,
                       const int64_t* y_strides, int32_t inverse, void* stream) {
  HF_TRY(check_type(dtype, head_dim));
  HF_TRY(check_rope(rope, head_dim));
  if (batch < 1 || batch > 65535 || heads < 1 || heads > 65535) { set_error("batch and heads must be in [1, 65535]"); return HF_ERR_SHAPE; }
  HF_TRY(check_rows(n_tokens, "n_tokens"));
  if (n_tokens == 0) return HF_OK;
  View x = {};
  x.dims = 3;
  x.n[0] = batch;
  x.n[1] = heads;
  x.n[2] = n_tokens;
  x.row = head_dim;
  x.es = dtype == HF_BF16 ? 2 : 4;
  View y = x;
  const int64_t defaults[3] = {(int64_t)heads * n_tokens * head_dim, (int64_t)n_tokens * head_dim, head_dim};
  HF_TRY(check_view(x, X, "X", x_strides, defaults, false));
  HF_TRY(check_ptr(positions, "positions", 4));
  HF_TRY(check_view(y, Y, "Y", y_strides, defaults, true));
  HF_TRY(check_apart(x, y, "Y overlaps X without being X", true));
  if (overlap(positions, (int64_t)(positions_per_batch ? batch : 1) * rope->n_axes * n_tokens * 4, y.p, y.span())) {
    set_error("Y overlaps positions");
    return HF_ERR_SHAPE;
  }
  return launch_rope_axes(*rope, dtype, head_dim, batch, heads, n_tokens, X, x.stride, positions, positions_per_batch != 0, Y, y.stride,
                          inverse != 0, static_cast<hipStream_t>(stream));
}

int hf_paged_append(const hf_paged* cache, const hf_rope_axes* rope_or_null, int32_t n_new, const void* K_new, const int64_t* k_strides,
                    const void* V_new, const int64_t* v_strides, const void* Q_or_null, const int64_t* q_strides, const int32_t* cu_new,
                    const int32_t* seq_lens, const int32_t* positions, void* K_pages, void* V_pages, const int32_t* page_table, void* Q_out,
                    const int64_t* q_out_strides, void* stream) {
  HF_TRY(check_cache(cache));
  if (rope_or_null) HF_TRY(check_rope(rope_or_null, cache->head_dim));
  HF_TRY(check_rows(n_new, "n_new"));
  if ((Q_or_null == nullptr) != (Q_out == nullptr)) { set_error("Q and Q_out must both be given or both be NULL"); return HF_ERR_NULL; }
  if (n_new == 0) return HF_OK;
  View k = packed(*cache, n_new, cache->heads_kv), v = k, q = packed(*cache, n_new, cache->heads), o = q;
  HF_TRY(check_packed(k, K_new, "K_new", k_strides, false));
  HF_TRY(check_packed(v, V_new, "V_new", v_strides, false));
  HF_TRY(check_pool(cache, K_pages, V_pages, page_table, cu_new, seq_lens));
  if (positions) HF_TRY(check_ptr(positions, "positions", 4));
  const int64_t pool = pool_bytes(*cache);
  if (overlap(K_pages, pool, V_pages, pool)) { set_error("K_pages overlaps V_pages"); return HF_ERR_SHAPE; }
  for (const View* x : {&k, &v})
    if (overlap(x->p, x->span(), K_pages, pool) || overlap(x->p, x->span(), V_pages, pool)) {
      set_error("%s overlaps the pages", x == &k ? "K_new" : "V_new");
      return HF_ERR_SHAPE;
    }
  const int32_t* read = rope_or_null ? positions : nullptr;
  const int64_t n_read = rope_or_null ? (int64_t)rope_or_null->n_axes * n_new : 0;
  HF_TRY(check_reads(K_pages, pool, "K_pages", *cache, cu_new, seq_lens, page_table, read, n_read));
  HF_TRY(check_reads(V_pages, pool, "V_pages", *cache, cu_new, seq_lens, page_table, read, n_read));
  if (Q_or_null) {
    HF_TRY(check_packed(q, Q_or_null, "Q", q_strides, false));
    HF_TRY(check_packed(o, Q_out, "Q_out", q_out_strides, true));
    HF_TRY(check_apart(q, o, "Q_out overlaps Q without being Q", true));
    for (const View* x : {&q, &o})
      if (overlap(x->p, x->span(), K_pages, pool) || overlap(x->p, x->span(), V_pages, pool)) {
        set_error("%s overlaps the pages", x == &q ? "Q" : "Q_out");
        return HF_ERR_SHAPE;
      }
    HF_TRY(check_reads(o.p, o.span(), "Q_out", *cache, cu_new, seq_lens, page_table, read, n_read));
  }
  return launch_paged_append(*cache, rope_or_null, n_new, K_new, k.stride, V_new, v.stride, Q_or_null, q.stride, cu_new, seq_lens, positions,
                             K_pages, V_pages, page_table, Q_out, o.stride, static_cast<hipStream_t>(stream));
}

int hf_paged_workspace_bytes(const hf_paged* cache, int32_t n_q, size_t* bytes_out) {
  HF_TRY(check_cache(cache));
  if (!bytes_out) { set_error("bytes_out is NULL"); return HF_ERR_NULL; }
  HF_TRY(check_attn_rows(cache, n_q));
  *bytes_out = paged_workspace_bytes(*cache, n_q);
  return HF_OK;
}

int hf_paged_attn_fwd(const hf_paged* cache, const void* Q, const int64_t* q_strides, int32_t n_q, const int32_t* cu_new,
                      const int32_t* seq_lens, const void* K_pages, const void* V_pages, const int32_t* page_table, void* O,
                      const int64_t* o_strides, float* lse2_or_null, void* workspace, size_t workspace_bytes, void* stream) {
  HF_TRY(check_cache(cache));
  HF_TRY(check_attn_rows(cache, n_q));
  if (n_q == 0) return HF_OK;
  View q = packed(*cache, n_q, cache->heads), o = q;
  HF_TRY(check_packed(q, Q, "Q", q_strides, false));
  HF_TRY(check_pool(cache, K_pages, V_pages, page_table, cu_new, seq_lens));
  HF_TRY(check_packed(o, O, "O", o_strides, true));
  HF_TRY(check_apart(q, o, "O overlaps Q", false));
  const int64_t pool = pool_bytes(*cache), lse = lse2_or_null ? (int64_t)cache->heads * n_q * 4 : 0;
  if (overlap(o.p, o.span(), K_pages, pool) || overlap(o.p, o.span(), V_pages, pool)) { set_error("O overlaps the pages"); return HF_ERR_SHAPE; }
  HF_TRY(check_reads(o.p, o.span(), "O", *cache, cu_new, seq_lens, page_table));
  if (lse2_or_null) {
    HF_TRY(check_ptr(lse2_or_null, "lse2", 4));
    if (overlap(o.p, o.span(), lse2_or_null, lse) || overlap(q.p, q.span(), lse2_or_null, lse) || overlap(K_pages, pool, lse2_or_null, lse) ||
        overlap(V_pages, pool, lse2_or_null, lse)) {
      set_error("lse2 overlaps another argument");
      return HF_ERR_SHAPE;
    }
    HF_TRY(check_reads(lse2_or_null, lse, "lse2", *cache, cu_new, seq_lens, page_table));
  }
  const size_t need = paged_workspace_bytes(*cache, n_q);
  if (need) {
    if (!workspace || workspace_bytes < need) {
      set_error("workspace of %zu bytes needed, got %zu", need, workspace ? workspace_bytes : (size_t)0);
      return HF_ERR_WORKSPACE;
    }
    HF_TRY(check_ptr(workspace, "workspace", 256));
    const int64_t w = (int64_t)need;
    if (overlap(workspace, w, o.p, o.span()) || overlap(workspace, w, q.p, q.span()) || overlap(workspace, w, K_pages, pool) ||
        overlap(workspace, w, V_pages, pool) || (lse && overlap(workspace, w, lse2_or_null, lse))) {
      set_error("workspace overlaps another argument");
      return HF_ERR_SHAPE;
    }
    HF_TRY(check_reads(workspace, w, "workspace", *cache, cu_new, seq_lens, page_table));
  }
  PagedAttnArgs a = {};
  a.Q = Q;
  a.K_pages = K_pages;
  a.V_pages = V_pages;
  a.O = O;
  a.cu = cu_new;
  a.lens = seq_lens;
  a.table = page_table;
  a.lse2 = lse2_or_null;
  a.qt = q.stride[0];
  a.qh = q.stride[1];
  a.ot = o.stride[0];
  a.oh = o.stride[1];
  a.n_q = n_q;
  a.heads = cache->heads;
  a.heads_kv = cache->heads_kv;
  a.page = cache->page_tokens;
  a.n_pages = cache->n_pages;
  a.n_seqs = cache->n_seqs;
  a.max_pages = cache->max_pages;
  a.causal = cache->causal != 0;
  a.window = cache->window;
  a.n_sink = cache->n_sink;
  a.c_scale = (cache->softmax_scale > 0.0f ? cache->softmax_scale : 1.0f / sqrtf((float)cache->head_dim)) * 1.44269504088896340736f;
  return launch_paged_attn(*cache, a, workspace, static_cast<hipStream_t>(stream));
}

}  // extern "C"
