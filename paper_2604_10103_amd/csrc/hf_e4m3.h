// Norms with rotation, and the cache of pages in 8 bits: launchers behind their entry points (internal).
#pragma once

#include "hf_paged.h"

namespace hf {

int launch_norm_rope(const hf_head_norm* norm, const hf_rope_axes* r, const hf_rope_scaling* sc, int dtype, int D, int batch, int heads, int n,
                     const void* X, const int64_t* xs, const float* weight, const int32_t* positions, bool per_batch, void* Y,
                     const int64_t* ys, hipStream_t s);
size_t norm_rope_bwd_workspace_bytes(int D, int batch, int heads, int n, bool per_head);
int launch_norm_rope_bwd(const hf_head_norm* norm, const hf_rope_axes* r, const hf_rope_scaling* sc, int dtype, int D, int batch, int heads,
                         int n, const void* X, const int64_t* xs, const float* weight, const int32_t* positions, bool per_batch,
                         const void* dY, const int64_t* gs, void* dX, const int64_t* ds, float* dweight, void* workspace, hipStream_t s);
int launch_append_e4m3(const hf_paged& c, const hf_head_norm* norm, const hf_rope_axes* r, const hf_rope_scaling* sc, int n, const void* K,
                       const int64_t* ks, const void* V, const int64_t* vs, const void* Q, const int64_t* qs, const float* k_weight,
                       const float* q_weight, const int32_t* cu, const int32_t* lens, const int32_t* positions, void* K_pages, void* V_pages,
                       float* K_scales, float* V_scales, const int32_t* table, void* Q_out, const int64_t* os, hipStream_t s);

long long paged_e4m3_threads(const hf_paged& c, int n_q);   // of the launch; 2^32 are too many
size_t paged_e4m3_workspace_bytes(const hf_paged& c, int n_q);
int launch_paged_attn_e4m3(const hf_paged& c, PagedAttnArgs a, const float* K_scales, const float* V_scales, void* workspace, hipStream_t s);

}  // namespace hf
