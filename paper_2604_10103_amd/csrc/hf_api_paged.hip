// Entry points of the rotation by positions and of the cache of pages: host-side argument checks, then the launch.
#include <math.h>

#include "hf_api_checks.h"
#include "hf_paged.h"

using namespace hf;

namespace {

int check_attn_rows(const hf_paged* c, int32_t n_q) {
  HF_TRY(check_rows(n_q, "n_q"));
  if ((int64_t)n_q * c->heads > (1ll << 30)) { set_error("n_q * heads must be <= 2^30"); return HF_ERR_SHAPE; }
  if (n_q > 0 && paged_threads(*c, n_q) >= (1ll << 32)) { set_error("more rows and sequences than a launch of 2^32 threads holds"); return HF_ERR_SHAPE; }
  return HF_OK;
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
    HF_TRY(check_queries_apart(o, k, v));
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
