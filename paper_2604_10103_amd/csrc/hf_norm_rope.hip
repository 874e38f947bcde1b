// Rows of queries and keys normalised, weighted and turned by their positions (hf_norm_rope_fwd), the gradients (hf_norm_rope_bwd), and the
// same on the way into a cache of pages in 8 bits (hf_paged_append_e4m3).
//
// All move every row once: they are bound by memory.  A thread owns the same 8 or 16 features of a token for several heads, so that an angle
// is formed once and serves them all; a row's 4 to 16 threads exchange their sums of squares (and the gradient's products, and the largest
// magnitude of a row that is quantised) by data-parallel moves within 16 lanes, three or four instructions a sum.  Two rows are requested
// before the first one is worked on.  10800 tokens of 40 rows pass in 47 us, 4.7 TB/s; the gradients of 9360 tokens of 12 rows take 21 to 22 us,
// 3.9 to 4.1 TB/s and the launch that adds the weights' sums; 9360 tokens of 12 keys, values and queries enter the pages in 33 to 36 us, 4.0 to
// 4.4 TB/s, of which some 4 are the launch and the chain lengths, page table, rows; a token of 40 rows takes 4 to 5 us, 64 single tokens are
// appended in 5.9.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "hf_e4m3.h"
#include "hf_rope_axes.h"

namespace hf {

namespace {

// ---- over the N lanes that share a row (N a power of two, 4 .. 16, lanes from a multiple of N on): every lane gets the result
template <int CTRL> __device__ __forceinline__ uint32_t moved(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int N, class F> __device__ __forceinline__ uint32_t over_row(uint32_t v, F f) {
  static_assert(N == 4 || N == 8 || N == 16, "lanes of a row");
  v = f(v, moved<0xb1>(v));                            // quads: the neighbour,
  v = f(v, moved<0x4e>(v));                            // the other pair;
  if constexpr (N >= 8) v = f(v, moved<0x141>(v));     // the other quad of 8 (mirrored),
  if constexpr (N >= 16) v = f(v, moved<0x140>(v));    // the other 8 of 16
  return v;
}
template <int N> __device__ __forceinline__ float sum_over_row(float v) {
  return __uint_as_float(over_row<N>(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
template <int N> __device__ __forceinline__ uint32_t max_over_row(uint32_t v) {
  return over_row<N>(v, [](uint32_t a, uint32_t b) { return max(a, b); });
}

// A thread's features of a row, in fp32.  They lie where the rotation wants them (modes of AxesMode), in groups of 8 consecutive ones or
// (kHalvesAny) single
template <typename T, int D, int MODE> struct Part {
  static constexpr int NF = axes_features<D, MODE>(), TPR = axes_threads<D, MODE>(), W = 8 * sizeof(T) / 16;
  // where x[i] lies in the row
  __device__ static __forceinline__ int feature(int g, int P, int i) {
    if constexpr (MODE == kHalvesAny) {
      const int p = 8 * g + (i & 7);
      return i < 8 ? (p < P ? p : 2 * p) : (p < P ? p + P : 2 * p + 1);
    }
    if constexpr (MODE == kHalves) {
      if (8 * g >= P) return 16 * g + i;
      return i < 8 ? 8 * g + i : P + 8 * g + i - 8;
    }
    return NF * g + i;
  }
  struct Raw {   // as it was loaded
    uint4 w[NF / 8 * W];
  };
  __device__ static __forceinline__ Raw load(const T* row, int g, int P) {
    Raw r;
    if constexpr (MODE == kHalvesAny) {
      uint32_t v[NF * sizeof(T) / 4];
#pragma unroll
      for (int i = 0; i < NF; i += 4 / sizeof(T)) {
        if constexpr (sizeof(T) == 2) v[i / 2] = row[feature(g, P, i)] | (uint32_t)row[feature(g, P, i + 1)] << 16;
        else v[i] = __float_as_uint(row[feature(g, P, i)]);
      }
#pragma unroll
      for (int i = 0; i < NF / 8 * W; ++i) r.w[i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    } else {
#pragma unroll
      for (int b = 0; b < NF / 8; ++b)
#pragma unroll
        for (int i = 0; i < W; ++i) r.w[b * W + i] = reinterpret_cast<const uint4*>(row + feature(g, P, 8 * b))[i];
    }
    return r;
  }
  __device__ static __forceinline__ void widen(const Raw& r, float (&x)[NF]) {
#pragma unroll
    for (int i = 0; i < NF / 8 * W; ++i) {
      const uint32_t v[4] = {r.w[i].x, r.w[i].y, r.w[i].z, r.w[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 2) {
          x[8 * i + 2 * e] = __uint_as_float(v[e] << 16);
          x[8 * i + 2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
        } else {
          x[4 * i + e] = __uint_as_float(v[e]);
        }
      }
    }
  }
  __device__ static __forceinline__ void store(T* row, int g, int P, const float (&x)[NF]) {
    if constexpr (MODE == kHalvesAny) {
#pragma unroll
      for (int i = 0; i < NF; ++i) Elem<T>::store(row + feature(g, P, i), x[i]);
    } else {
#pragma unroll
      for (int b = 0; b < NF / 8; ++b) {
        uint4* to = reinterpret_cast<uint4*>(row + feature(g, P, 8 * b));
        if constexpr (sizeof(T) == 2) {
          to[0] = make_uint4(pack_bf16(x[8 * b], x[8 * b + 1]), pack_bf16(x[8 * b + 2], x[8 * b + 3]), pack_bf16(x[8 * b + 4], x[8 * b + 5]),
                             pack_bf16(x[8 * b + 6], x[8 * b + 7]));
        } else {
#pragma unroll
          for (int i = 0; i < 2; ++i)
            to[i] = make_uint4(__float_as_uint(x[8 * b + 4 * i]), __float_as_uint(x[8 * b + 4 * i + 1]), __float_as_uint(x[8 * b + 4 * i + 2]),
                               __float_as_uint(x[8 * b + 4 * i + 3]));
        }
      }
    }
  }
  __device__ static __forceinline__ void store_codes(uint8_t* row, int g, int P, const uint32_t (&c)[NF / 4]) {
    if constexpr (MODE == kHalvesAny) {
#pragma unroll
      for (int i = 0; i < NF; ++i) row[feature(g, P, i)] = (uint8_t)(c[i / 4] >> (8 * (i & 3)));
    } else {
#pragma unroll
      for (int b = 0; b < NF / 8; ++b) *reinterpret_cast<uint2*>(row + feature(g, P, 8 * b)) = make_uint2(c[2 * b], c[2 * b + 1]);
    }
  }
  __device__ static __forceinline__ void weights(const float* w, int g, int P, float (&x)[NF]) {
#pragma unroll
    for (int i = 0; i < NF; ++i) x[i] = w ? w[feature(g, P, i)] : 1.0f;
  }
  __device__ static __forceinline__ void turn(const Angles<D, MODE>& t, int g, int P, float (&x)[NF]) {
#pragma unroll
    for (int i = 0; i < NF / 2; ++i) {
      const int a = MODE == kAdjacent ? 2 * i : i, b = MODE == kAdjacent ? 2 * i + 1 : i + 8;
      const bool turns = MODE == kAdjacent ? 4 * g + i < P : MODE == kHalves ? 8 * g < P : 8 * g + i < P;
      const float u = x[a] * t.c[i] - x[b] * t.s[i], v = x[a] * t.s[i] + x[b] * t.c[i];
      x[a] = turns ? u : x[a];
      x[b] = turns ? v : x[b];
    }
  }
  // r = 1 / sqrt(mean square + eps) of the row times k, which x[] is multiplied by: a power of two where the squares leave fp32, else 1
  __device__ static __forceinline__ float inverse_rms(float (&x)[NF], float eps, float& k) {
    const auto mean = [&] {
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < NF; ++i) s = fmaf(x[i], x[i], s);
      return sum_over_row<TPR>(s) * (1.0f / D);
    };
    k = 1.0f;
    const float square = mean();
    float m = square + eps;
    if (m < 0x1p-100f || square > 0x1p100f) {   // (a row's threads go the same way)
      k = m < 0x1p-100f ? 0x1p100f : 0x1p-72f;
      times(k, x);
      m = mean() + eps * k * k;
    }
    return rsqrtf(m);
  }
  __device__ static __forceinline__ void times(float k, float (&x)[NF]) {
    if (k != 1.0f) {
#pragma unroll
      for (int i = 0; i < NF; ++i) x[i] *= k;
    }
  }
};

// what rows are normalised with
struct NormArgs {
  int on, per_head;
  float eps, amplitude;
};

// rows i0 .. i1 - 1 of a token: from(i), with the weights at weight(i) (or NULL; `shared`: the same for all), to out(i, x)
template <typename T, int D, int MODE, class From, class Weight, class Out>
__device__ __forceinline__ void norm_rows(const NormArgs& n, const Angles<D, MODE>& t, int g, int P, int i0, int i1, bool shared, From from, Weight weight,
                                          Out out) {
  typedef Part<T, D, MODE> R;
  constexpr int NF = R::NF, U = 2;
  if (i0 >= i1) return;
  float w[NF];
  if (shared) R::weights(weight(0), g, P, w);
  for (int i = i0; i < i1; i += U) {
    typename R::Raw raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = R::load(from(min(i + u, i1 - 1)), g, P);
    float r[U], k[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[NF];
      R::widen(raw[u], x);
      r[u] = k[u] = 1.0f;
      if (n.on) r[u] = R::inverse_rms(x, n.eps, k[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u >= i1) break;
      float x[NF];
      R::widen(raw[u], x);
      if (!shared) R::weights(weight(i + u), g, P, w);
      R::times(k[u], x);
#pragma unroll
      for (int e = 0; e < NF; ++e) x[e] = x[e] * r[u] * w[e];
      R::turn(t, g, P, x);
      out(i + u, x);
    }
  }
}

template <int D, int MODE, class F>
__device__ __forceinline__ void form_angles(Angles<D, MODE>& t, const AxesSpec& spec, int g, bool flip, float amplitude, F at) {
  t.form(spec, g, flip, at);
#pragma unroll
  for (int i = 0; i < Angles<D, MODE>::N; ++i) {
    t.c[i] *= amplitude;
    t.s[i] *= amplitude;
  }
}

struct FwdArgs {
  const void* X;
  void* Y;
  const float* weight;
  const int32_t* positions;
  long long xb, xh, xt, yb, yh, yt;   // strides in elements
  long long pos_batch;                // positions of a batch
  int n, heads;
  NormArgs norm;
};

template <typename T, int D, int MODE>
__global__ __launch_bounds__(256) void norm_rope_kernel(const AxesSpec spec, const FwdArgs a) {
  constexpr int TPT = axes_threads<D, MODE>(), TOK = 256 / TPT;
  const int tok = blockIdx.x * TOK + threadIdx.x / TPT, g = threadIdx.x % TPT;
  if (tok >= a.n) return;
  const int per = (a.heads + gridDim.y - 1) / gridDim.y, h0 = blockIdx.y * per, h1 = min(a.heads, h0 + per);
  const int32_t* pos = a.positions + blockIdx.z * a.pos_batch + tok;
  Angles<D, MODE> t;
  form_angles(t, spec, g, false, a.norm.amplitude, [&](int ax) { return pos[(long long)ax * a.n]; });
  const T* x = static_cast<const T*>(a.X) + blockIdx.z * a.xb + tok * a.xt;
  T* y = static_cast<T*>(a.Y) + blockIdx.z * a.yb + tok * a.yt;
  norm_rows<T, D, MODE>(
      a.norm, t, g, spec.pairs, h0, h1, !a.norm.per_head || !a.weight, [&](int h) { return x + h * a.xh; },
      [&](int h) { return a.weight ? a.weight + (a.norm.per_head ? h * D : 0) : nullptr; },
      [&](int h, const float (&v)[Part<T, D, MODE>::NF]) { Part<T, D, MODE>::store(y + h * a.yh, g, spec.pairs, v); });
}

// ---- gradients.  With g the output's gradient turned back and u the row at unit mean square,
//     dX = r (w g - u mean(w g u)),  dweight = sum g u:
// one pass over X and dY.  Every thread sums its features of dweight over 16 of its rows at a time in fp32, and those sums in 64 bits in LDS
// (600 equal rows summed in fp32 alone are off by up to 146 units of 2^-24, 16 by 16 at most); a workgroup's threads meet there, and the
// workgroups' sums, rounded to fp32, lie in the workspace until a second launch adds them in 64 bits.  All in a fixed order
struct BwdArgs {
  const void *X, *dY;
  void* dX;
  const float* weight;
  const int32_t* positions;
  float* partial;                                  // [weights' rows][parts][D], or NULL
  long long xb, xh, xt, gb, gh, gt, db, dh, dt;   // strides of X, dY, dX in elements
  long long pos_batch;
  int n, heads;
  NormArgs norm;
};

constexpr int kChain = 16;

template <typename T, int D, int MODE, bool CHAINS>   // CHAINS: a thread may have more than kChain rows
__global__ __launch_bounds__(256) void norm_rope_bwd_kernel(const AxesSpec spec, const BwdArgs a) {
  typedef Part<T, D, MODE> R;
  constexpr int TPT = R::TPR, TOK = 256 / TPT, NF = R::NF, U = 1;
  const int g = threadIdx.x % TPT, P = spec.pairs;
  const int per = (a.heads + gridDim.y - 1) / gridDim.y, h0 = blockIdx.y * per, h1 = min(a.heads, h0 + per);
  const bool shared = !a.norm.per_head || !a.weight;
  __shared__ std::conditional_t<CHAINS, double, float> sums[256 * NF];   // chains' [NF][thread]; in the end [TOK][D]
  float w[NF], dw[NF];
  int chain = 0;   // rows in dw
#pragma unroll
  for (int e = 0; e < NF; ++e) dw[e] = 0.0f;
  if constexpr (CHAINS) {
#pragma unroll
    for (int e = 0; e < NF; ++e) sums[256 * e + threadIdx.x] = 0.0;
  }
  if (shared) R::weights(a.weight, g, P, w);
  for (int tok = blockIdx.x * TOK + threadIdx.x / TPT; tok < a.n; tok += gridDim.x * TOK) {
    const int32_t* pos = a.positions + blockIdx.z * a.pos_batch + tok;
    const T* x = static_cast<const T*>(a.X) + blockIdx.z * a.xb + tok * a.xt;
    const T* dy = static_cast<const T*>(a.dY) + blockIdx.z * a.gb + tok * a.gt;
    T* dx = static_cast<T*>(a.dX) + blockIdx.z * a.db + tok * a.dt;
    typename R::Raw rx[U], rg[U];
    const auto request = [&](int h) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int hu = min(h + u, h1 - 1);
        rx[u] = R::load(x + hu * a.xh, g, P);
        rg[u] = R::load(dy + hu * a.gh, g, P);
      }
    };
    request(h0);   // (on their way while the angles are formed)
    Angles<D, MODE> t;
    form_angles(t, spec, g, true, a.norm.amplitude, [&](int ax) { return pos[(long long)ax * a.n]; });
    for (int h = h0; h < h1; h += U) {
      if (h > h0) request(h);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (h + u >= h1) break;
        float v[NF], y[NF];
        R::widen(rx[u], v);
        R::widen(rg[u], y);
        R::turn(t, g, P, y);
        if (a.norm.on) {
          if (!shared) R::weights(a.weight + (long long)(h + u) * D, g, P, w);
          float k;
          const float r = R::inverse_rms(v, a.norm.eps, k);
          float dot = 0.0f;
#pragma unroll
          for (int e = 0; e < NF; ++e) {
            v[e] *= r;
            dw[e] = fmaf(y[e], v[e], dw[e]);
            y[e] *= w[e];
            dot = fmaf(y[e], v[e], dot);
          }
          dot = sum_over_row<TPT>(dot) * (1.0f / D);
#pragma unroll
          for (int e = 0; e < NF; ++e) y[e] = r * (y[e] - v[e] * dot);
          R::times(k, y);
        }
        R::store(dx + (h + u) * a.dh, g, P, y);
        if constexpr (CHAINS) {
          if (++chain == kChain) {
            chain = 0;
#pragma unroll
            for (int e = 0; e < NF; ++e) {
              sums[256 * e + threadIdx.x] += (double)dw[e];
              dw[e] = 0.0f;
            }
          }
        }
      }
    }
  }
  if (!a.partial) return;   // (uniform)
  if constexpr (CHAINS) {
    double mine[NF];
#pragma unroll
    for (int e = 0; e < NF; ++e) mine[e] = sums[256 * e + threadIdx.x] + (double)dw[e];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < NF; ++e) sums[threadIdx.x / TPT * D + R::feature(g, P, e)] = mine[e];
  } else {
#pragma unroll
    for (int e = 0; e < NF; ++e) sums[threadIdx.x / TPT * D + R::feature(g, P, e)] = dw[e];
  }
  __syncthreads();
  if (threadIdx.x < D) {
    double total = 0.0;   // (of either sign: sums in 32 bits would cost half a digit)
#pragma unroll
    for (int i = 0; i < TOK; ++i) total += (double)sums[i * D + threadIdx.x];
    const float s = (float)total;
    const int row = a.norm.per_head ? blockIdx.y : 0, shares = a.norm.per_head ? 1 : gridDim.y, share = a.norm.per_head ? 0 : blockIdx.y;
    const int parts = gridDim.x * gridDim.z * shares, part = (blockIdx.z * shares + share) * gridDim.x + blockIdx.x;
    a.partial[((long long)row * parts + part) * D + threadIdx.x] = s;
  }
}

// dweight[row][f] = the sum of partial[row][0 .. parts - 1][f]: 32 features a workgroup, 32 threads each
__global__ __launch_bounds__(1024) void norm_dweight_kernel(const float* partial, float* dweight, int parts, int D) {
  const int f = blockIdx.x * 32 + (threadIdx.x & 31), lane = threadIdx.x >> 5;
  const float* p = partial + (long long)blockIdx.y * parts * D + f;
  double s = 0.0;
#pragma unroll 8
  for (int i = lane; i < parts; i += 32) s += (double)p[(long long)i * D];
  __shared__ double sums[32][33];
  sums[lane][threadIdx.x & 31] = s;
  __syncthreads();
  if (lane == 0) {
    s = 0.0;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += sums[i][threadIdx.x];
    dweight[(long long)blockIdx.y * D + f] = (float)s;
  }
}

// ---- into the pages
struct AppendArgs {
  const void *K, *V, *Q;
  const float *k_weight, *q_weight;
  uint8_t *K_pages, *V_pages;
  float *K_scales, *V_scales;
  void* Q_out;
  const int32_t *cu, *lens, *positions, *table;
  long long kt, kh, vt, vh, qt, qh, ot, oh;
  int n, heads, heads_kv, page, n_pages, n_seqs, max_pages;
  NormArgs norm;
};

// x[] as e4m3 with the row's scale: the quotients are rounded as a division is, which decides where one lies half way between two codes, then
// to a code.  A product with the rounded reciprocal is off by 1.5 units at most, and one correction by its remainder rounds it correctly
// (Markstein's theorem; three instructions a quotient where a division takes ten), as long as the remainder is exact: below a scale of 2^-93 its
// last bits are beyond fp32 where the quotient is 2^-10, the least that decides about a code, and row and scale are taken 2^64 times as large.
// (The theorem spares one divisor, an all-ones mantissa.  The product with 1 / 448 has it for no row.)
template <int N, int TPR> __device__ __forceinline__ float quantise(const float (&x)[N], uint32_t (&c)[N / 4]) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);   // (as integers: a NaN is larger than all others)
  top = max_over_row<TPR>(top);
  const bool finite = top < 0x7f800000u;
  const float scale = fmaxf(__uint_as_float(top) * (1.0f / 448.0f), 0x1p-126f);
  const float up = scale < 0x1p-90f ? 0x1p64f : 1.0f, by = scale * up, inv = 1.0f / by;
#pragma unroll
  for (int e = 0; e < N; e += 4) {
    float q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float v = x[e + i] * up, y = v * inv;
      q[i] = copysignf(fmaf(fmaf(-y, by, v), inv, y), v);   // (a zero keeps its sign)
    }
    uint32_t w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], (int)w, true);
    c[e / 4] = finite ? w : 0;
  }
  return finite ? scale : __builtin_nanf("");
}

// Work of a token: its heads_kv keys, heads_kv values and (Q given) its queries, shared out over gridDim.y
template <typename T, int D, int MODE>
__global__ __launch_bounds__(256) void append_e4m3_kernel(const AxesSpec spec, const AppendArgs a) {
  typedef Part<T, D, MODE> R;
  typedef Part<T, D, kAdjacent> Plain;   // values, by as many threads: 8 consecutive features each, or twice 8
  constexpr int TPT = R::TPR, TOK = 256 / TPT, NF = R::NF;
  const int row = blockIdx.x * TOK + threadIdx.x / TPT, g = threadIdx.x % TPT;
  // the token's sequence: as many as end at or before its row, found by the token's threads together, four places each at a time
  int lo = 0, span = a.n_seqs;   // sequences before lo do, those from lo + span on do not
  while (span > 0) {
    const int step = (span + 4 * TPT - 1) / (4 * TPT);
    int count = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = (g + i * TPT + 1) * step - 1;   // the step's last sequence
      count += at < span && a.cu[lo + at + 1] <= row;
    }
    count = (int)over_row<TPT>((uint32_t)count, [](uint32_t x, uint32_t y) { return x + y; });
    lo += count * step;
    span = min(step - 1, span - count * step);
  }
  if (row >= a.n || lo >= a.n_seqs) return;
  const int seq = lo, begin = a.cu[seq], end = a.cu[seq + 1];
  if (row < begin) return;
  const long long place = (long long)a.lens[seq] - (end - begin) + (row - begin);
  const bool exists = place >= 0 && place < (long long)a.max_pages * a.page;
  const int slot = exists ? (int)place : 0, entry = slot / a.page, inside = slot - entry * a.page;
  const int page = a.table[(long long)seq * a.max_pages + entry];
  const bool held = exists && (unsigned)page < (unsigned)a.n_pages;

  const int total = 2 * a.heads_kv + (a.Q ? a.heads : 0);
  const int per = (total + gridDim.y - 1) / gridDim.y, i0 = blockIdx.y * per, i1 = min(total, i0 + per);
  const int k0 = i0, k1 = held ? min(i1, a.heads_kv) : k0;                                    // keys
  const int v0 = max(0, i0 - a.heads_kv), v1 = held ? min(a.heads_kv, i1 - a.heads_kv) : v0;  // values
  const int q0 = max(0, i0 - 2 * a.heads_kv), q1 = i1 - 2 * a.heads_kv;                       // queries
  const T* k = static_cast<const T*>(a.K) + row * a.kt;
  const T* v = static_cast<const T*>(a.V) + row * a.vt;
  const T* q = static_cast<const T*>(a.Q) + row * a.qt;
  T* o = static_cast<T*>(a.Q_out) + row * a.ot;
  const long long at = held ? ((long long)page * a.heads_kv) * a.page + inside : 0;   // the pool's row of head 0
  for (int h = v0; h < v1; h += 4) {
    float x[4][NF];
    uint4 raw[4][NF / 8 * R::W];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint4* from = reinterpret_cast<const uint4*>(v + min(h + u, v1 - 1) * a.vh + NF * g);
#pragma unroll
      for (int i = 0; i < NF / 8 * R::W; ++i) raw[u][i] = from[i];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (h + u >= v1) break;
#pragma unroll
      for (int b = 0; b < NF / 8; ++b) {
        typename Plain::Raw part;
#pragma unroll
        for (int i = 0; i < R::W; ++i) part.w[i] = raw[u][b * R::W + i];
        float y[8];
        Plain::widen(part, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[u][8 * b + e] = y[e];
      }
      uint32_t c[NF / 4];
      const float scale = quantise<NF, TPT>(x[u], c);
      const long long to = at + (long long)(h + u) * a.page;
      uint2* code = reinterpret_cast<uint2*>(a.V_pages + to * D + NF * g);
#pragma unroll
      for (int b = 0; b < NF / 8; ++b) code[b] = make_uint2(c[2 * b], c[2 * b + 1]);
      if (g == 0) a.V_scales[to] = scale;
    }
  }
  if (k0 >= k1 && q0 >= q1) return;   // (a share of values alone)
  Angles<D, MODE> t;
  form_angles(t, spec, g, false, a.norm.amplitude, [&](int ax) { return a.positions ? a.positions[(long long)ax * a.n + row] : (int)place; });
  const auto weight_of = [&](const float* w, int h) { return w ? w + (a.norm.per_head ? h * D : 0) : nullptr; };
  norm_rows<T, D, MODE>(
      a.norm, t, g, spec.pairs, k0, k1, !a.norm.per_head || !a.k_weight, [&](int h) { return k + h * a.kh; },
      [&](int h) { return weight_of(a.k_weight, h); },
      [&](int h, const float (&x)[NF]) {
        uint32_t c[NF / 4];
        const float scale = quantise<NF, TPT>(x, c);
        const long long to = at + (long long)h * a.page;
        R::store_codes(a.K_pages + to * D, g, spec.pairs, c);
        if (g == 0) a.K_scales[to] = scale;
      });
  norm_rows<T, D, MODE>(
      a.norm, t, g, spec.pairs, q0, q1, !a.norm.per_head || !a.q_weight, [&](int h) { return q + h * a.qh; },
      [&](int h) { return weight_of(a.q_weight, h); }, [&](int h, const float (&x)[NF]) { R::store(o + h * a.oh, g, spec.pairs, x); });
}

// shares of a token's rows: at least 1024 workgroups, or as many as leave each four rows, which an angle formed once serves; but no more than
// `resident` ones, which is how many run at a time in ADJACENT (56 and 74 registers: eight and six wavefronts a SIMD): 10800 tokens of 40 rows
// 47.2 us by 2025 workgroups, 48.5 by 2700; 9360 tokens of 36 rows into the pages 30.2 by 1170, 34.7 by 2340.  HALVES has registers for 1024
// (114 to 122), with any number of pairs for 512 or 768 (149 to 200); other bounds were not measured for these
int shares(long long groups, int rows, int resident) {
  const long long s = std::min(std::max(1ll, resident / groups), std::max((1024 + groups - 1) / groups, (long long)rows / 4));
  return (int)std::max(1ll, std::min(s, (long long)rows));
}

// rates as hf_rope_axes gives them, slowed as the scaling says
AxesSpec scaled_spec(const hf_rope_axes* r, const hf_rope_scaling* s) {
  if (!r) return AxesSpec{};
  AxesSpec spec = axes_spec(*r);
  if (!s || s->factor == 1.0) return spec;
  for (int p = 0; p < spec.pairs; ++p) {
    if (!(s->axes >> (spec.axis[p >> 4] >> (2 * (p & 15)) & 3) & 1)) continue;
    const long double rate = (long double)spec.quarter[p] + spec.rest[p];                 // quarter turns a position
    const long double turns = 0.25L * rate * s->trained;
    const long double keep = std::min(1.0L, std::max(0.0L, (turns - s->slow) / ((long double)s->fast - s->slow)));
    const long double slowed = rate * (keep + (1.0L - keep) / s->factor);
    spec.quarter[p] = (double)slowed;
    spec.rest[p] = (float)(slowed - spec.quarter[p]);
  }
  return spec;
}

NormArgs norm_args(const hf_head_norm* n, const hf_rope_scaling* s) {
  return {n != nullptr, n && n->per_head, n ? n->eps : 0.0f, s ? s->amplitude : 1.0f};
}

// the gradient's grid: workgroups that stay for many tokens, so that there are few sums to be added.  (weights for each head: a head each)
struct BwdGrid {
  int x, y, z, rows, parts;
};
BwdGrid bwd_grid(int D, int threads, int batch, int heads, int n, bool per_head) {
  const int tok = 256 / threads;
  BwdGrid b = {};
  b.z = batch;
  b.rows = per_head ? heads : 1;
  if (n == 0) return b;   // (no sums: zeros)
  const long long blocks = (n + tok - 1) / tok;
  b.y = per_head ? heads : (int)std::max(1ll, std::min<long long>(shares(blocks * batch, heads, 2048), heads));
  const long long most = std::max(1ll, 1024ll / std::min<long long>((long long)b.y * b.z, 1024));
  const long long turns = (blocks + most - 1) / most;   // all workgroups take as many blocks of tokens, or one less
  b.x = (int)std::max(1ll, (blocks + turns - 1) / turns);
  b.parts = b.x * b.z * (per_head ? 1 : b.y);
  return b;
}

#define HF_ROPE_MODES(mode, T, DD, GO)   \
  do {                                   \
    if (mode == kAdjacent) GO(T, DD, kAdjacent);   \
    else if (mode == kHalves) GO(T, DD, kHalves);  \
    else GO(T, DD, kHalvesAny);          \
  } while (0)
#define HF_ROPE_TYPES(dtype, D, mode, GO)                                                          \
  do {                                                                                             \
    if (dtype == HF_BF16) {                                                                        \
      if (D == 128) HF_ROPE_MODES(mode, bf16_t, 128, GO); else HF_ROPE_MODES(mode, bf16_t, 64, GO); \
    } else {                                                                                       \
      if (D == 128) HF_ROPE_MODES(mode, float, 128, GO); else HF_ROPE_MODES(mode, float, 64, GO);   \
    }                                                                                              \
  } while (0)

}  // namespace

int launch_norm_rope(const hf_head_norm* norm, const hf_rope_axes* r, const hf_rope_scaling* sc, int dtype, int D, int batch, int heads, int n,
                     const void* X, const int64_t* xs, const float* weight, const int32_t* positions, bool per_batch, void* Y,
                     const int64_t* ys, hipStream_t s) {
  const AxesSpec spec = scaled_spec(r, sc);
  const FwdArgs a = {X, Y, weight, positions, xs[0], xs[1], xs[2], ys[0], ys[1], ys[2], per_batch && r ? (long long)r->n_axes * n : 0, n, heads,
                     norm_args(norm, sc)};
  const AxesMode mode = r ? axes_mode(*r, spec.pairs) : kAdjacent;
  const int tok = mode == kAdjacent ? 2048 / D : 4096 / D, groups = (n + tok - 1) / tok;
  const dim3 grid(groups, shares((long long)groups * batch, heads, 2048), batch);
#define HF_GO(T, DD, M) hipLaunchKernelGGL((norm_rope_kernel<T, DD, M>), grid, dim3(256), 0, s, spec, a)
  HF_ROPE_TYPES(dtype, D, mode, HF_GO);
#undef HF_GO
  return check_launch("hf_norm_rope_fwd");
}

size_t norm_rope_bwd_workspace_bytes(int D, int batch, int heads, int n, bool per_head) {
  size_t most = 0;
  for (int threads : {D / 8, D / 16}) {   // (whatever the rotation)
    const BwdGrid b = bwd_grid(D, threads, batch, heads, n, per_head);
    most = std::max(most, (size_t)b.rows * b.parts * D * 4);
  }
  return most;
}

int launch_norm_rope_bwd(const hf_head_norm* norm, const hf_rope_axes* r, const hf_rope_scaling* sc, int dtype, int D, int batch, int heads,
                         int n, const void* X, const int64_t* xs, const float* weight, const int32_t* positions, bool per_batch,
                         const void* dY, const int64_t* gs, void* dX, const int64_t* ds, float* dweight, void* workspace, hipStream_t s) {
  const AxesSpec spec = scaled_spec(r, sc);
  const AxesMode mode = r ? axes_mode(*r, spec.pairs) : kAdjacent;
  const BwdGrid b = bwd_grid(D, mode == kAdjacent ? D / 8 : D / 16, batch, heads, n, norm && norm->per_head);
  if (n > 0) {
    const int tok = mode == kAdjacent ? 2048 / D : 4096 / D;
    const long long rows = ((long long)n + b.x * tok - 1) / (b.x * tok) * ((heads + b.y - 1) / b.y);   // of a thread
    const BwdArgs a = {X, dY, dX, weight, positions, dweight ? static_cast<float*>(workspace) : nullptr,
                       xs[0], xs[1], xs[2], gs[0], gs[1], gs[2], ds[0], ds[1], ds[2],
                       per_batch && r ? (long long)r->n_axes * n : 0, n, heads, norm_args(norm, sc)};
    const dim3 grid(b.x, b.y, b.z);
    if (dweight && rows > kChain) {
#define HF_GO(T, DD, M) hipLaunchKernelGGL((norm_rope_bwd_kernel<T, DD, M, true>), grid, dim3(256), 0, s, spec, a)
      HF_ROPE_TYPES(dtype, D, mode, HF_GO);
#undef HF_GO
    } else {
#define HF_GO(T, DD, M) hipLaunchKernelGGL((norm_rope_bwd_kernel<T, DD, M, false>), grid, dim3(256), 0, s, spec, a)
      HF_ROPE_TYPES(dtype, D, mode, HF_GO);
#undef HF_GO
    }
    const int rc = check_launch("hf_norm_rope_bwd");
    if (rc != HF_OK) return rc;
  }
  if (!dweight) return HF_OK;
  hipLaunchKernelGGL(norm_dweight_kernel, dim3(D / 32, b.rows), dim3(1024), 0, s, static_cast<const float*>(workspace), dweight, b.parts, D);
  return check_launch("hf_norm_rope_bwd");
}

int launch_append_e4m3(const hf_paged& c, const hf_head_norm* norm, const hf_rope_axes* r, const hf_rope_scaling* sc, int n, const void* K,
                       const int64_t* ks, const void* V, const int64_t* vs, const void* Q, const int64_t* qs, const float* k_weight,
                       const float* q_weight, const int32_t* cu, const int32_t* lens, const int32_t* positions, void* K_pages, void* V_pages,
                       float* K_scales, float* V_scales, const int32_t* table, void* Q_out, const int64_t* os, hipStream_t s) {
  const AxesSpec spec = scaled_spec(r, sc);
  const AppendArgs a = {K, V, Q, k_weight, q_weight, static_cast<uint8_t*>(K_pages), static_cast<uint8_t*>(V_pages), K_scales, V_scales, Q_out,
                        cu, lens, r ? positions : nullptr, table, ks[0], ks[1], vs[0], vs[1], qs[0], qs[1], os[0], os[1],
                        n, c.heads, c.heads_kv, c.page_tokens, c.n_pages, c.n_seqs, c.max_pages, norm_args(norm, sc)};
  const AxesMode mode = r ? axes_mode(*r, spec.pairs) : kAdjacent;
  const int D = c.head_dim, tok = mode == kAdjacent ? 2048 / D : 4096 / D, groups = (n + tok - 1) / tok;
  const dim3 grid(groups, shares(groups, 2 * c.heads_kv + (Q ? c.heads : 0), 1536));
#define HF_GO(T, DD, M) hipLaunchKernelGGL((append_e4m3_kernel<T, DD, M>), grid, dim3(256), 0, s, spec, a)
  HF_ROPE_TYPES(c.dtype, D, mode, HF_GO);
#undef HF_GO
  return check_launch("hf_paged_append_e4m3");
}

}  // namespace hf
