// Entry points of the norms with rotation and of the cache of pages in 8 bits: host-side argument checks, then the launch.
#include "hf_api_checks.h"
#include "hf_e4m3.h"

using namespace hf;

namespace {

int check_norm(const hf_head_norm* n) {
  if (n && (!(n->eps >= 0.0f) || !isfinite(n->eps))) { set_error("eps must be finite and >= 0"); return HF_ERR_SHAPE; }
  return HF_OK;
}

int check_scaling(const hf_rope_scaling* s, const hf_rope_axes* r) {
  if (!s) return HF_OK;
  if (!r) { set_error("scaling without rope"); return HF_ERR_NULL; }
  if (!(s->factor >= 1.0) || !isfinite(s->factor)) { set_error("factor must be finite and >= 1"); return HF_ERR_SHAPE; }
  if (!(s->trained > 0.0) || !isfinite(s->trained)) { set_error("trained must be finite and > 0"); return HF_ERR_SHAPE; }
  if (!(s->slow >= 0.0) || !(s->fast > s->slow) || !isfinite(s->fast)) { set_error("slow and fast must be finite, 0 <= slow < fast"); return HF_ERR_SHAPE; }
  if (!(s->amplitude > 0.0f) || !isfinite(s->amplitude)) { set_error("amplitude must be finite and > 0"); return HF_ERR_SHAPE; }
  if (s->axes < 0 || s->axes >> r->n_axes) { set_error("axes names an axis that the rope does not have"); return HF_ERR_SHAPE; }
  return HF_OK;
}

// Memory that a call is given, as a list: what it writes lies over none of the rest
struct Span {
  const void* p;
  int64_t bytes;
  const char* name;
};

int check_written(const Span* written, int n_written, const Span* read, int n_read) {
  for (int i = 0; i < n_written; ++i) {
    if (!written[i].p) continue;
    for (int j = 0; j < n_read; ++j)
      if (read[j].p && overlap(written[i].p, written[i].bytes, read[j].p, read[j].bytes)) {
        set_error("%s overlaps %s", written[i].name, read[j].name);
        return HF_ERR_SHAPE;
      }
    for (int j = 0; j < i; ++j)
      if (written[j].p && overlap(written[i].p, written[i].bytes, written[j].p, written[j].bytes)) {
        set_error("%s overlaps %s", written[i].name, written[j].name);
        return HF_ERR_SHAPE;
      }
  }
  return HF_OK;
}

Span span_of(const View& v, const char* name) { return {v.p, v.p ? v.span() : 0, name}; }

// what both directions of norm and rotation check before their operands
int check_norm_rope(const hf_head_norm* norm, const hf_rope_axes* rope, const hf_rope_scaling* scaling, int32_t dtype, int32_t head_dim,
                    int32_t batch, int32_t heads, int32_t n_tokens) {
  HF_TRY(check_type(dtype, head_dim));
  HF_TRY(check_norm(norm));
  if (rope) HF_TRY(check_rope(rope, head_dim));
  if (!norm && !rope) { set_error("neither norm nor rope"); return HF_ERR_NULL; }
  HF_TRY(check_scaling(scaling, rope));
  if (batch < 1 || batch > 65535 || heads < 1 || heads > 65535) { set_error("batch and heads must be in [1, 65535]"); return HF_ERR_SHAPE; }
  return check_rows(n_tokens, "n_tokens");
}

struct RowOperands {
  View x, y, dx;
  Span weight, positions;
};

RowOperands row_operands(int dtype, int head_dim, int batch, int heads, int n_tokens) {
  RowOperands o = {};
  o.x.dims = 3;
  o.x.n[0] = batch;
  o.x.n[1] = heads;
  o.x.n[2] = n_tokens;
  o.x.row = head_dim;
  o.x.es = dtype == HF_BF16 ? 2 : 4;
  o.y = o.dx = o.x;
  return o;
}

int check_extras(RowOperands& o, const hf_head_norm* norm, const hf_rope_axes* rope, int head_dim, int batch, int heads, int n_tokens,
                 const float* weight, const int32_t* positions, int per_batch) {
  if (weight && !norm) { set_error("weight without norm"); return HF_ERR_NULL; }
  if (weight) HF_TRY(check_ptr(weight, "weight", 4));
  if (rope) HF_TRY(check_ptr(positions, "positions", 4));
  o.weight = {weight, (int64_t)(norm && norm->per_head ? heads : 1) * head_dim * 4, "weight"};
  o.positions = {rope ? positions : nullptr, rope ? (int64_t)(per_batch ? batch : 1) * rope->n_axes * n_tokens * 4 : 0, "positions"};
  return HF_OK;
}

int check_e4m3_attn_rows(const hf_paged* c, int32_t n_q) {
  HF_TRY(check_rows(n_q, "n_q"));
  if ((int64_t)n_q * c->heads > (1ll << 30)) { set_error("n_q * heads must be <= 2^30"); return HF_ERR_SHAPE; }
  if (n_q > 0 && paged_e4m3_threads(*c, n_q) >= (1ll << 32)) { set_error("more rows and sequences than a launch of 2^32 threads holds"); return HF_ERR_SHAPE; }
  return HF_OK;
}

int64_t pool_rows(const hf_paged& c) { return (int64_t)c.n_pages * c.heads_kv * c.page_tokens; }

int check_scales(const float* k, const float* v) {
  HF_TRY(check_ptr(k, "K_scales", 4));
  return check_ptr(v, "V_scales", 4);
}

}  // namespace

extern "C" {

int hf_norm_rope_fwd(const hf_head_norm* norm_or_null, const hf_rope_axes* rope_or_null, const hf_rope_scaling* scaling_or_null, int32_t dtype,
                     int32_t head_dim, int32_t batch, int32_t heads, int32_t n_tokens, const void* X, const int64_t* x_strides,
                     const float* weight_or_null, const int32_t* positions, int32_t positions_per_batch, void* Y, const int64_t* y_strides,
                     void* stream) {
  HF_TRY(check_norm_rope(norm_or_null, rope_or_null, scaling_or_null, dtype, head_dim, batch, heads, n_tokens));
  if (n_tokens == 0) return HF_OK;
  RowOperands o = row_operands(dtype, head_dim, batch, heads, n_tokens);
  const int64_t defaults[3] = {(int64_t)heads * n_tokens * head_dim, (int64_t)n_tokens * head_dim, head_dim};
  HF_TRY(check_view(o.x, X, "X", x_strides, defaults, false));
  HF_TRY(check_extras(o, norm_or_null, rope_or_null, head_dim, batch, heads, n_tokens, weight_or_null, positions, positions_per_batch));
  HF_TRY(check_view(o.y, Y, "Y", y_strides, defaults, true));
  HF_TRY(check_apart(o.x, o.y, "Y overlaps X without being X", true));
  const Span written = span_of(o.y, "Y"), read[] = {o.weight, o.positions};
  HF_TRY(check_written(&written, 1, read, 2));
  return launch_norm_rope(norm_or_null, rope_or_null, scaling_or_null, dtype, head_dim, batch, heads, n_tokens, X, o.x.stride, weight_or_null,
                          positions, positions_per_batch != 0, Y, o.y.stride, static_cast<hipStream_t>(stream));
}

int hf_norm_rope_bwd_workspace_bytes(const hf_head_norm* norm, int32_t head_dim, int32_t batch, int32_t heads, int32_t n_tokens,
                                     size_t* bytes_out) {
  if (!norm) { set_error("norm is NULL"); return HF_ERR_NULL; }
  HF_TRY(check_norm_rope(norm, nullptr, nullptr, HF_F32, head_dim, batch, heads, n_tokens));
  if (!bytes_out) { set_error("bytes_out is NULL"); return HF_ERR_NULL; }
  *bytes_out = norm_rope_bwd_workspace_bytes(head_dim, batch, heads, n_tokens, norm->per_head != 0);
  return HF_OK;
}

int hf_norm_rope_bwd(const hf_head_norm* norm_or_null, const hf_rope_axes* rope_or_null, const hf_rope_scaling* scaling_or_null, int32_t dtype,
                     int32_t head_dim, int32_t batch, int32_t heads, int32_t n_tokens, const void* X, const int64_t* x_strides,
                     const float* weight_or_null, const int32_t* positions, int32_t positions_per_batch, const void* dY,
                     const int64_t* dy_strides, void* dX, const int64_t* dx_strides, float* dweight_or_null, void* workspace,
                     size_t workspace_bytes, void* stream) {
  HF_TRY(check_norm_rope(norm_or_null, rope_or_null, scaling_or_null, dtype, head_dim, batch, heads, n_tokens));
  if (dweight_or_null && !norm_or_null) { set_error("dweight without norm"); return HF_ERR_NULL; }
  if (n_tokens == 0 && !dweight_or_null) return HF_OK;
  RowOperands o = row_operands(dtype, head_dim, batch, heads, n_tokens);
  const int64_t defaults[3] = {(int64_t)heads * n_tokens * head_dim, (int64_t)n_tokens * head_dim, head_dim};
  if (n_tokens > 0) {
    HF_TRY(check_view(o.x, X, "X", x_strides, defaults, false));
    HF_TRY(check_extras(o, norm_or_null, rope_or_null, head_dim, batch, heads, n_tokens, weight_or_null, positions, positions_per_batch));
    HF_TRY(check_view(o.y, dY, "dY", dy_strides, defaults, false));
    HF_TRY(check_view(o.dx, dX, "dX", dx_strides, defaults, true));
    HF_TRY(check_apart(o.x, o.dx, "dX overlaps X without being X", true));
    HF_TRY(check_apart(o.y, o.dx, "dX overlaps dY without being dY", true));
  }
  Span ws = {nullptr, 0, "workspace"};
  if (dweight_or_null) {
    HF_TRY(check_ptr(dweight_or_null, "dweight", 4));
    const size_t need = norm_rope_bwd_workspace_bytes(head_dim, batch, heads, n_tokens, norm_or_null->per_head != 0);
    if (need) {
      if (!workspace || workspace_bytes < need) {
        set_error("workspace of %zu bytes needed, got %zu", need, workspace ? workspace_bytes : (size_t)0);
        return HF_ERR_WORKSPACE;
      }
      HF_TRY(check_ptr(workspace, "workspace", 256));
      ws = {workspace, (int64_t)need, "workspace"};
    }
  }
  const Span written[] = {{o.dx.p, o.dx.p ? o.dx.span() : 0, "dX"},
                          {dweight_or_null, (int64_t)(norm_or_null && norm_or_null->per_head ? heads : 1) * head_dim * 4, "dweight"},
                          ws};
  const Span read[] = {o.weight, o.positions};
  HF_TRY(check_written(written, 3, read, 2));
  const Span rows[] = {span_of(o.x, "X"), span_of(o.y, "dY")};
  HF_TRY(check_written(written + 1, 2, rows, 2));
  return launch_norm_rope_bwd(norm_or_null, rope_or_null, scaling_or_null, dtype, head_dim, batch, heads, n_tokens, X, o.x.stride, weight_or_null,
                              positions, positions_per_batch != 0, dY, o.y.stride, dX, o.dx.stride, dweight_or_null, workspace,
                              static_cast<hipStream_t>(stream));
}

int hf_paged_append_e4m3(const hf_paged* cache, const hf_head_norm* norm_or_null, const hf_rope_axes* rope_or_null,
                         const hf_rope_scaling* scaling_or_null, int32_t n_new, const void* K_new, const int64_t* k_strides, const void* V_new,
                         const int64_t* v_strides, const void* Q_or_null, const int64_t* q_strides, const float* k_weight_or_null,
                         const float* q_weight_or_null, const int32_t* cu_new, const int32_t* seq_lens, const int32_t* positions, void* K_pages,
                         void* V_pages, float* K_scales, float* V_scales, const int32_t* page_table, void* Q_out, const int64_t* q_out_strides,
                         void* stream) {
  HF_TRY(check_cache(cache));
  HF_TRY(check_norm(norm_or_null));
  if (rope_or_null) HF_TRY(check_rope(rope_or_null, cache->head_dim));
  HF_TRY(check_scaling(scaling_or_null, rope_or_null));
  HF_TRY(check_rows(n_new, "n_new"));
  if ((Q_or_null == nullptr) != (Q_out == nullptr)) { set_error("Q and Q_out must both be given or both be NULL"); return HF_ERR_NULL; }
  if ((k_weight_or_null || q_weight_or_null) && !norm_or_null) { set_error("weights without norm"); return HF_ERR_NULL; }
  if (n_new == 0) return HF_OK;
  View k = packed(*cache, n_new, cache->heads_kv), v = k, q = packed(*cache, n_new, cache->heads), o = q;
  HF_TRY(check_packed(k, K_new, "K_new", k_strides, false));
  HF_TRY(check_packed(v, V_new, "V_new", v_strides, false));
  HF_TRY(check_pool(cache, K_pages, V_pages, page_table, cu_new, seq_lens));
  HF_TRY(check_scales(K_scales, V_scales));
  if (positions) HF_TRY(check_ptr(positions, "positions", 4));
  if (k_weight_or_null) HF_TRY(check_ptr(k_weight_or_null, "k_weight", 4));
  if (q_weight_or_null) HF_TRY(check_ptr(q_weight_or_null, "q_weight", 4));
  if (Q_or_null) {
    HF_TRY(check_packed(q, Q_or_null, "Q", q_strides, false));
    HF_TRY(check_packed(o, Q_out, "Q_out", q_out_strides, true));
    HF_TRY(check_apart(q, o, "Q_out overlaps Q without being Q", true));
  }
  const bool each = norm_or_null && norm_or_null->per_head;
  const int64_t rows = pool_rows(*cache), w = 4ll * cache->head_dim;
  const Span written[] = {{K_pages, rows * cache->head_dim, "K_pages"}, {V_pages, rows * cache->head_dim, "V_pages"},
                          {K_scales, rows * 4, "K_scales"}, {V_scales, rows * 4, "V_scales"}, span_of(o, "Q_out")};
  const Span read[] = {span_of(k, "K_new"), span_of(v, "V_new"), {cu_new, 4ll * (cache->n_seqs + 1), "cu_new"},
                       {seq_lens, 4ll * cache->n_seqs, "seq_lens"}, {page_table, 4ll * cache->n_seqs * cache->max_pages, "page_table"},
                       {rope_or_null ? positions : nullptr, rope_or_null ? 4ll * rope_or_null->n_axes * n_new : 0, "positions"},
                       {k_weight_or_null, w * (each ? cache->heads_kv : 1), "k_weight"}, {q_weight_or_null, w * (each ? cache->heads : 1), "q_weight"},
                       span_of(q, "Q")};
  HF_TRY(check_written(written, 4, read, 9));
  HF_TRY(check_written(written + 4, 1, read + 2, 6));
  if (o.p) HF_TRY(check_queries_apart(o, k, v));
  for (int i = 0; i < 4; ++i)
    if (o.p && overlap(o.p, o.span(), written[i].p, written[i].bytes)) { set_error("Q_out overlaps %s", written[i].name); return HF_ERR_SHAPE; }
  return launch_append_e4m3(*cache, norm_or_null, rope_or_null, scaling_or_null, n_new, K_new, k.stride, V_new, v.stride, Q_or_null, q.stride,
                            k_weight_or_null, q_weight_or_null, cu_new, seq_lens, positions, K_pages, V_pages, K_scales, V_scales, page_table,
                            Q_out, o.stride, static_cast<hipStream_t>(stream));
}

int hf_paged_e4m3_workspace_bytes(const hf_paged* cache, int32_t n_q, size_t* bytes_out) {
  HF_TRY(check_cache(cache));
  if (!bytes_out) { set_error("bytes_out is NULL"); return HF_ERR_NULL; }
  HF_TRY(check_e4m3_attn_rows(cache, n_q));
  *bytes_out = paged_e4m3_workspace_bytes(*cache, n_q);
  return HF_OK;
}

int hf_paged_attn_e4m3_fwd(const hf_paged* cache, const void* Q, const int64_t* q_strides, int32_t n_q, const int32_t* cu_new,
                           const int32_t* seq_lens, const void* K_pages, const void* V_pages, const float* K_scales, const float* V_scales,
                           const int32_t* page_table, void* O, const int64_t* o_strides, float* lse2_or_null, void* workspace,
                           size_t workspace_bytes, void* stream) {
  HF_TRY(check_cache(cache));
  HF_TRY(check_e4m3_attn_rows(cache, n_q));
  if (n_q == 0) return HF_OK;
  View q = packed(*cache, n_q, cache->heads), o = q;
  HF_TRY(check_packed(q, Q, "Q", q_strides, false));
  HF_TRY(check_pool(cache, K_pages, V_pages, page_table, cu_new, seq_lens));
  HF_TRY(check_scales(K_scales, V_scales));
  HF_TRY(check_packed(o, O, "O", o_strides, true));
  if (lse2_or_null) HF_TRY(check_ptr(lse2_or_null, "lse2", 4));
  const size_t need = paged_e4m3_workspace_bytes(*cache, n_q);
  if (need) {
    if (!workspace || workspace_bytes < need) {
      set_error("workspace of %zu bytes needed, got %zu", need, workspace ? workspace_bytes : (size_t)0);
      return HF_ERR_WORKSPACE;
    }
    HF_TRY(check_ptr(workspace, "workspace", 256));
  }
  const int64_t rows = pool_rows(*cache);
  const Span written[] = {span_of(o, "O"), {lse2_or_null, 4ll * cache->heads * n_q, "lse2"}, {need ? workspace : nullptr, (int64_t)need, "workspace"}};
  const Span read[] = {span_of(q, "Q"), {cu_new, 4ll * (cache->n_seqs + 1), "cu_new"}, {seq_lens, 4ll * cache->n_seqs, "seq_lens"},
                       {page_table, 4ll * cache->n_seqs * cache->max_pages, "page_table"}, {K_pages, rows * cache->head_dim, "K_pages"},
                       {V_pages, rows * cache->head_dim, "V_pages"}, {K_scales, rows * 4, "K_scales"}, {V_scales, rows * 4, "V_scales"}};
  HF_TRY(check_written(written, 3, read, 8));
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
  return launch_paged_attn_e4m3(*cache, a, K_scales, V_scales, workspace, static_cast<hipStream_t>(stream));
}

}  // extern "C"
