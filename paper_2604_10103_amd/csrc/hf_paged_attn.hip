// Attention of packed new tokens over a cache of pages: one wavefront per row and head.
#include "hf_paged.h"

namespace hf {

namespace {

template <typename T, int D>
__global__ __launch_bounds__(256) void paged_attn_kernel(const PagedAttnArgs a) {
  const int lane = threadIdx.x & 63;
  const long long item = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (item >= (long long)a.n_q * a.heads) return;
  const int row = (int)(item / a.heads), head = (int)(item % a.heads), hk = head / (a.heads / a.heads_kv);
  int seq = 0;
  for (int j = lane; j < a.n_seqs; j += kWave) seq += a.cu[j + 1] <= row;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) seq += __shfl_xor(seq, o, kWave);
  if (seq >= a.n_seqs || row < a.cu[seq]) return;
  const long long most = (long long)a.max_pages * a.page;
  const long long len = a.lens[seq], p = len - (a.cu[seq + 1] - a.cu[seq]) + (row - a.cu[seq]);
  const long long end = max(0ll, min(min(len, most), a.causal ? p + 1 : len));
  const long long first = a.window > 0 ? max(0ll, p - a.window + 1) : 0;
  const T* q = static_cast<const T*>(a.Q) + row * a.qt + head * a.qh;
  float m = -INFINITY, l = 0.0f, o[D / 64];
  bool any = false;
#pragma unroll
  for (int f = 0; f < D / 64; ++f) o[f] = 0.0f;
  for (long long j0 = 0; j0 < end; j0 += kWave) {
    const long long j = j0 + lane;
    bool sees = j < end && (j >= first || j < a.n_sink);
    long long at = 0;
    if (sees) {
      const int page = a.table[(long long)seq * a.max_pages + j / a.page];
      sees = (unsigned)page < (unsigned)a.n_pages;
      at = (((long long)page * a.heads_kv + hk) * a.page + j % a.page) * D;
    }
    float s = -INFINITY;
    if (sees) {
      s = 0.0f;
      const T* k = static_cast<const T*>(a.K_pages) + at;
      for (int f = 0; f < D; ++f) s = fmaf(Elem<T>::load(q + f), Elem<T>::load(k + f), s);
      s *= a.c_scale;
    }
    unsigned long long see = __ballot(sees);
    if (see == 0) continue;
    any = true;
    const float m_new = fmaxf(m, wave_max(s)), m_use = m_new == -INFINITY ? 0.0f : m_new;
    const float w = __builtin_amdgcn_exp2f(m - m_use);
    const float pr = sees ? __builtin_amdgcn_exp2f(s - m_use) : 0.0f;
    l = l * w + wave_sum(pr);
    m = m_new;
#pragma unroll
    for (int f = 0; f < D / 64; ++f) o[f] *= w;
    for (; see; see &= see - 1) {
      const int src = __ffsll(see) - 1;
      const T* v = static_cast<const T*>(a.V_pages) + __shfl(at, src, kWave);
      const float pk = __shfl(pr, src, kWave);
#pragma unroll
      for (int f = 0; f < D / 64; ++f) o[f] = fmaf(pk, Elem<T>::load(v + 64 * f + lane), o[f]);
    }
  }
  T* out = static_cast<T*>(a.O) + row * a.ot + head * a.oh;
#pragma unroll
  for (int f = 0; f < D / 64; ++f) Elem<T>::store(out + 64 * f + lane, any ? o[f] / l : 0.0f);
  if (a.lse2 && lane == 0) a.lse2[(long long)head * a.n_q + row] = any ? m + log2f(l) : INFINITY;
}

}  // namespace

size_t paged_workspace_bytes(const hf_paged&, int) { return 0; }

int launch_paged_attn(const hf_paged& c, const PagedAttnArgs& a, void*, hipStream_t s) {
  const unsigned grid = (unsigned)(((long long)a.n_q * a.heads + 3) / 4);
#define HF_LAUNCH_PAGED(T, DD) hipLaunchKernelGGL((paged_attn_kernel<T, DD>), dim3(grid), dim3(256), 0, s, a)
  if (c.dtype == HF_BF16) {
    if (c.head_dim == 128) HF_LAUNCH_PAGED(bf16_t, 128); else HF_LAUNCH_PAGED(bf16_t, 64);
  } else {
    if (c.head_dim == 128) HF_LAUNCH_PAGED(float, 128); else HF_LAUNCH_PAGED(float, 64);
  }
#undef HF_LAUNCH_PAGED
  return check_launch("hf_paged_attn_fwd");
}

}  // namespace hf
