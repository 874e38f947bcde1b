// Rows turned by positions with several axes (hf_rope_axes_apply), and the same on the way into a cache of pages (hf_paged_append).
//
// Both move every row once: they are bound by memory.  A thread owns the same few pairs of a token for many heads, so that an angle
// (a product and a reduction in 64 bits, two polynomials: some fifty instructions) is formed once and serves them all.  10800 tokens of
// 80 rows turn in 89 us, 5.0 TB/s; two streams' 4680 tokens of 12 keys, values and queries are appended in 42 us, 4.1 TB/s, of which some
// 4 us are the launch and the chain lengths, page table, rows; a token of 40 rows turns in 4 to 4.7 us, 64 single tokens are appended in 5.7.
#include <math.h>

#include <algorithm>

#include "hf_paged.h"
#include "hf_rope_axes.h"

namespace hf {

namespace {

struct ApplyArgs {
  const void* X;
  void* Y;
  const int32_t* positions;
  long long xb, xh, xt, yb, yh, yt;   // strides in elements
  long long pos_batch;                // positions of a batch
  int n, heads, flip;
};

template <typename T, int D, int MODE>
__global__ __launch_bounds__(256) void rope_axes_kernel(const AxesSpec spec, const ApplyArgs a) {
  constexpr int TPT = axes_threads<D, MODE>(), TOK = 256 / TPT;
  const int tok = blockIdx.x * TOK + threadIdx.x / TPT, g = threadIdx.x % TPT;
  if (tok >= a.n) return;
  const int per = (a.heads + gridDim.y - 1) / gridDim.y, h0 = blockIdx.y * per, h1 = min(a.heads, h0 + per);
  const int32_t* pos = a.positions + blockIdx.z * a.pos_batch + tok;
  Angles<D, MODE> t;
  t.form(spec, g, a.flip, [&](int ax) { return pos[(long long)ax * a.n]; });
  const T* x = static_cast<const T*>(a.X) + blockIdx.z * a.xb + tok * a.xt;
  T* y = static_cast<T*>(a.Y) + blockIdx.z * a.yb + tok * a.yt;
  turn_rows<T, D, MODE>(t, g, spec.pairs, h0, h1, [&](int h) { return x + h * a.xh; }, [&](int h) { return y + h * a.yh; });
}

struct AppendArgs {
  const void *K, *V, *Q;
  void *K_pages, *V_pages, *Q_out;
  const int32_t *cu, *lens, *positions, *table;
  long long kt, kh, vt, vh, qt, qh, ot, oh;
  int n, heads, heads_kv, page, n_pages, n_seqs, max_pages;
};

// Work of a token: its heads_kv keys, heads_kv values and (Q given) its queries, shared out over gridDim.y
template <typename T, int D, int MODE, bool kRope>
__global__ __launch_bounds__(256) void paged_append_kernel(const AxesSpec spec, const AppendArgs a) {
  constexpr int TPT = axes_threads<D, MODE>(), TOK = 256 / TPT;
  const int row = blockIdx.x * TOK + threadIdx.x / TPT, g = threadIdx.x % TPT;
  // the token's sequence: as many as end at or before its row, counted by the token's threads together
  int seq = 0;
  for (int j = g; j < a.n_seqs; j += TPT) seq += a.cu[j + 1] <= row;
#pragma unroll
  for (int o = 1; o < TPT; o <<= 1) seq += __shfl_xor(seq, o, kWave);
  if (row >= a.n || seq >= a.n_seqs) return;
  const int begin = a.cu[seq], end = a.cu[seq + 1];
  if (row < begin) return;
  const long long place = (long long)a.lens[seq] - (end - begin) + (row - begin);
  const bool exists = place >= 0 && place < (long long)a.max_pages * a.page;
  const int slot = exists ? (int)place : 0, entry = slot / a.page, inside = slot - entry * a.page;
  const int page = a.table[(long long)seq * a.max_pages + entry];
  const bool held = exists && (unsigned)page < (unsigned)a.n_pages;

  const int total = 2 * a.heads_kv + (a.Q ? a.heads : 0);
  const int per = (total + gridDim.y - 1) / gridDim.y, i0 = blockIdx.y * per, i1 = min(total, i0 + per);
  const T* k = static_cast<const T*>(a.K) + row * a.kt;
  const T* v = static_cast<const T*>(a.V) + row * a.vt;
  const T* q = static_cast<const T*>(a.Q) + row * a.qt;
  T* o = static_cast<T*>(a.Q_out) + row * a.ot;
  const long long at = held ? (((long long)page * a.heads_kv) * a.page + inside) * D : 0;
  T* kp = static_cast<T*>(a.K_pages) + at;
  T* vp = static_cast<T*>(a.V_pages) + at;
  const long long ph = (long long)a.page * D;
  const int k0 = i0, k1 = held ? min(i1, a.heads_kv) : k0;                                    // keys
  const int v0 = max(0, i0 - a.heads_kv), v1 = held ? min(a.heads_kv, i1 - a.heads_kv) : v0;  // values
  const int q0 = max(0, i0 - 2 * a.heads_kv), q1 = i1 - 2 * a.heads_kv;                       // queries
  const auto k_from = [&](int h) { return k + h * a.kh; };
  const auto k_to = [&](int h) { return kp + h * ph; };
  const auto q_from = [&](int h) { return q + h * a.qh; };
  const auto q_to = [&](int h) { return o + h * a.oh; };
  copy_rows<T, D, MODE>(g, v0, v1, [&](int h) { return v + h * a.vh; }, [&](int h) { return vp + h * ph; });
  if constexpr (kRope) {
    if (k0 >= k1 && q0 >= q1) return;   // (a share of values alone)
    Angles<D, MODE> t;
    t.form(spec, g, false, [&](int ax) { return a.positions ? a.positions[(long long)ax * a.n + row] : (int)place; });
    turn_rows<T, D, MODE>(t, g, spec.pairs, k0, k1, k_from, k_to);
    turn_rows<T, D, MODE>(t, g, spec.pairs, q0, q1, q_from, q_to);
  } else {
    copy_rows<T, D, MODE>(g, k0, k1, k_from, k_to);
    copy_rows<T, D, MODE>(g, q0, q1, q_from, q_to);
  }
}

// shares of a token's rows: 2048 workgroups where that leaves each four rows, which are read together by an angle formed once (9360 tokens of
// 36 rows: 42 us, with 1024 workgroups 46), else 1024 (5121 tokens of 24 rows in fp32: 16.3 us, with 2048 19.2)
int shares(long long groups, int rows) {
  const auto for_groups = [&](int n) { return (n + groups - 1) / groups; };
  long long s = std::min(for_groups(2048), std::max(for_groups(1024), (long long)rows / 4));
  return (int)std::max(1ll, std::min(s, (long long)rows));
}

}  // namespace

int launch_rope_axes(const hf_rope_axes& r, int dtype, int D, int batch, int heads, int n, const void* X, const int64_t* xs,
                     const int32_t* positions, bool per_batch, void* Y, const int64_t* ys, bool inverse, hipStream_t s) {
  const AxesSpec spec = axes_spec(r);
  const ApplyArgs a = {X, Y, positions, xs[0], xs[1], xs[2], ys[0], ys[1], ys[2], per_batch ? (long long)r.n_axes * n : 0, n, heads, inverse};
  const AxesMode mode = axes_mode(r, spec.pairs);
  const int tok = mode == kAdjacent ? 2048 / D : 4096 / D, groups = (n + tok - 1) / tok;
  const dim3 grid(groups, shares((long long)groups * batch, heads), batch);
#define HF_LAUNCH_AXES(T, DD, M) hipLaunchKernelGGL((rope_axes_kernel<T, DD, M>), grid, dim3(256), 0, s, spec, a)
#define HF_LAUNCH_AXES_M(T, DD)                              \
  do {                                                       \
    if (mode == kAdjacent) HF_LAUNCH_AXES(T, DD, kAdjacent); \
    else if (mode == kHalves) HF_LAUNCH_AXES(T, DD, kHalves);\
    else HF_LAUNCH_AXES(T, DD, kHalvesAny);                  \
  } while (0)
  if (dtype == HF_BF16) {
    if (D == 128) HF_LAUNCH_AXES_M(bf16_t, 128); else HF_LAUNCH_AXES_M(bf16_t, 64);
  } else {
    if (D == 128) HF_LAUNCH_AXES_M(float, 128); else HF_LAUNCH_AXES_M(float, 64);
  }
#undef HF_LAUNCH_AXES_M
#undef HF_LAUNCH_AXES
  return check_launch("hf_rope_axes_apply");
}

int launch_paged_append(const hf_paged& c, const hf_rope_axes* r, int n, const void* K, const int64_t* ks, const void* V, const int64_t* vs,
                        const void* Q, const int64_t* qs, const int32_t* cu, const int32_t* lens, const int32_t* positions, void* K_pages,
                        void* V_pages, const int32_t* table, void* Q_out, const int64_t* os, hipStream_t s) {
  const AxesSpec spec = r ? axes_spec(*r) : AxesSpec{};
  const AppendArgs a = {K, V, Q, K_pages, V_pages, Q_out, cu, lens, positions, table, ks[0], ks[1], vs[0], vs[1], qs[0], qs[1], os[0], os[1],
                        n, c.heads, c.heads_kv, c.page_tokens, c.n_pages, c.n_seqs, c.max_pages};
  const AxesMode mode = r ? axes_mode(*r, spec.pairs) : kAdjacent;
  const int D = c.head_dim, tok = mode == kAdjacent ? 2048 / D : 4096 / D, groups = (n + tok - 1) / tok;
  const dim3 grid(groups, shares(groups, 2 * c.heads_kv + (Q ? c.heads : 0)));
#define HF_LAUNCH_APPEND(T, DD, M, R) hipLaunchKernelGGL((paged_append_kernel<T, DD, M, R>), grid, dim3(256), 0, s, spec, a)
#define HF_LAUNCH_APPEND_M(T, DD)                                       \
  do {                                                                  \
    if (!r) HF_LAUNCH_APPEND(T, DD, kAdjacent, false);                  \
    else if (mode == kAdjacent) HF_LAUNCH_APPEND(T, DD, kAdjacent, true); \
    else if (mode == kHalves) HF_LAUNCH_APPEND(T, DD, kHalves, true);   \
    else HF_LAUNCH_APPEND(T, DD, kHalvesAny, true);                     \
  } while (0)
  if (c.dtype == HF_BF16) {
    if (D == 128) HF_LAUNCH_APPEND_M(bf16_t, 128); else HF_LAUNCH_APPEND_M(bf16_t, 64);
  } else {
    if (D == 128) HF_LAUNCH_APPEND_M(float, 128); else HF_LAUNCH_APPEND_M(float, 64);
  }
#undef HF_LAUNCH_APPEND_M
#undef HF_LAUNCH_APPEND
  return check_launch("hf_paged_append");
}

}  // namespace hf
