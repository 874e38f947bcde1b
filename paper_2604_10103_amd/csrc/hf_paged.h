// The cache of pages: launchers behind its entry points (internal).
#pragma once

#include "hf_common.h"

namespace hf {

int launch_rope_axes(const hf_rope_axes& r, int dtype, int D, int batch, int heads, int n, const void* X, const int64_t* xs,
                     const int32_t* positions, bool per_batch, void* Y, const int64_t* ys, bool inverse, hipStream_t s);
int launch_paged_append(const hf_paged& c, const hf_rope_axes* r, int n, const void* K, const int64_t* ks, const void* V, const int64_t* vs,
                        const void* Q, const int64_t* qs, const int32_t* cu, const int32_t* lens, const int32_t* positions, void* K_pages,
                        void* V_pages, const int32_t* table, void* Q_out, const int64_t* os, hipStream_t s);

struct PagedAttnArgs {
  const void *Q, *K_pages, *V_pages;
  void* O;
  const int32_t *cu, *lens, *table;
  float* lse2;
  long long qt, qh, ot, oh;   // strides in elements
  int n_q, heads, heads_kv, group, page, n_pages, n_seqs, max_pages, causal, window, n_sink;
  float c_scale;              // softmax_scale * log2(e)
  uint32_t page_magic;        // key / page = key * page_magic >> page_shift for key < 2^31
  int page_shift;
  int page_tiles;             // > 0: key tiles end with their page, of which there are so many in one
  uint32_t tiles_magic;       // as above: tile / page_tiles, row / group (= heads / heads_kv)
  int tiles_shift;
  uint32_t group_magic;
  int group_shift;
};
long long paged_threads(const hf_paged& c, int n_q);   // of the launch; 2^32 are too many
size_t paged_workspace_bytes(const hf_paged& c, int n_q);
int launch_paged_attn(const hf_paged& c, PagedAttnArgs a, void* workspace, hipStream_t s);
struct PagedSchedule;
int launch_paged_attn_f32(const hf_paged& c, const PagedAttnArgs& a, const PagedSchedule& sc, int rows, int ks, int grid, hipStream_t s);

}  // namespace hf
