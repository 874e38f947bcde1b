// Rotation by positions with several axes: what the kernels that turn rows of head_dim features share (internal).
#pragma once

#include "hf_common.h"

namespace hf {

constexpr int kMaxPairs = 64;   // head_dim / 2

// by value in the kernels' arguments
struct AxesSpec {
  double quarter[kMaxPairs];   // quarter turns per position step of every pair,
  float rest[kMaxPairs];       // and what rounding to 64 bits left of them
  uint32_t axis[4];            // two bits a pair: its axis
  int pairs;                   // P
  int n_axes;
};

// how a row's pairs lie, and how its threads share them
enum AxesMode {
  kAdjacent = 0,   // pair p is (2p, 2p + 1): 8 consecutive features a thread
  kHalves = 1,     // (p, p + P), P a multiple of 8: 8 features of the first half and their partners a thread
  kHalvesAny = 2   // (p, p + P), any P: single elements, as a piece of one half and its partners in the other are not both aligned: 10800
                   // tokens of 80 rows in bf16 245 us (P = 61), where P a multiple of 8 takes 85
};

template <int D, int MODE> constexpr int axes_features() { return MODE == kAdjacent ? 8 : 16; }             // of a thread
template <int D, int MODE> constexpr int axes_threads() { return D / axes_features<D, MODE>(); }            // of a row

// cos and sin of pos * (quarter + rest) quarter turns.  In 64 bits the product alone would be off by 2^-22 of a radian at a position of
// 2^31, and so would the rate's rounding be: the whole quarter turns are taken from the product before it is rounded, and the rate's rest
// is added (in 32 bits a position of 2^16 would leave 2^-8).  What is left, [-1/2, 1/2] quarter turns, goes through the Taylor polynomials
// of degree 9 and 10, whose next terms are 1.8e-9 and 1.2e-10 at pi/4: 1.2 units of 2^-24 in all, at any position.
__device__ __forceinline__ void quarter_turns(double quarter, float rest, int pos, float& c, float& s) {
  const double x = (double)pos, q = rint(x * quarter), part = fma(x, (double)rest, fma(x, quarter, -q));
  const float a = (float)(part * 1.57079632679489661923), a2 = a * a;
  const int k = (int)q;   // (theta >= 1: below 2^31)
  const float sp = a * fmaf(a2, fmaf(a2, fmaf(a2, fmaf(a2, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f), 1.0f);
  const float cp = fmaf(a2, fmaf(a2, fmaf(a2, fmaf(a2, fmaf(a2, -1.0f / 3628800.0f, 1.0f / 40320.0f), -1.0f / 720.0f), 1.0f / 24.0f), -0.5f), 1.0f);
  const float u = (k & 1) ? sp : cp, v = (k & 1) ? cp : sp;
  c = ((k + 1) & 2) ? -u : u;
  s = (k & 2) ? -v : v;
}

// the angles of thread g of a token: 4 pairs (kAdjacent) or 8
template <int D, int MODE> struct Angles {
  static constexpr int N = axes_features<D, MODE>() / 2;
  float c[N], s[N];
  // at(a): the token's position on axis a; flip: the other way
  template <class F> __device__ __forceinline__ void form(const AxesSpec& spec, int g, bool flip, F at) {
    int pos[HF_ROPE_MAX_AXES];
#pragma unroll
    for (int a = 0; a < HF_ROPE_MAX_AXES; ++a) pos[a] = a < spec.n_axes ? at(a) : 0;
    double quarter[N];
    float rest[N];
    uint32_t axis = spec.axis[(N * g) >> 4] >> (2 * ((N * g) & 15));   // (N pairs lie in one word)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      quarter[i] = spec.quarter[N * g + i];
      rest[i] = spec.rest[N * g + i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int ax = (axis >> (2 * i)) & 3;
      const int p = ax < 2 ? (ax == 0 ? pos[0] : pos[1]) : (ax == 2 ? pos[2] : pos[3]);
      quarter_turns(quarter[i], rest[i], p, c[i], s[i]);
      if (flip) s[i] = -s[i];
    }
  }
};

// a thread's features of a row, as its storage type holds them
template <typename T, int D, int MODE> struct Piece16 {
  static constexpr int NF = axes_features<D, MODE>(), HALF = NF / 2;
  static constexpr int U = 8 * sizeof(T) / 16;   // 16-byte words of 8 features
  uint4 w[NF / 8 * U];

  // where the thread's features 0..7 and 8..15 lie in the row (kHalves: those behind the 2 P rotated ones follow each other)
  __device__ static __forceinline__ int first(int g, int P) { return MODE == kHalves && 8 * g >= P ? 16 * g : NF * g >> (MODE == kHalves); }
  __device__ static __forceinline__ int second(int g, int P) { return 8 * g < P ? P + 8 * g : 16 * g + 8; }

  __device__ __forceinline__ void load(const T* row, int g, int P) {
    const uint4* a = reinterpret_cast<const uint4*>(row + first(g, P));
#pragma unroll
    for (int i = 0; i < U; ++i) w[i] = a[i];
    if constexpr (NF == 16) {
      const uint4* b = reinterpret_cast<const uint4*>(row + second(g, P));
#pragma unroll
      for (int i = 0; i < U; ++i) w[U + i] = b[i];
    }
  }
  __device__ __forceinline__ void store(T* row, int g, int P) const {
    uint4* a = reinterpret_cast<uint4*>(row + first(g, P));
#pragma unroll
    for (int i = 0; i < U; ++i) a[i] = w[i];
    if constexpr (NF == 16) {
      uint4* b = reinterpret_cast<uint4*>(row + second(g, P));
#pragma unroll
      for (int i = 0; i < U; ++i) b[i] = w[U + i];
    }
  }
  // 16-byte words as they come, for rows that are copied
  __device__ __forceinline__ void load_plain(const T* row, int g) {
    const uint4* a = reinterpret_cast<const uint4*>(row + NF * g);
#pragma unroll
    for (int i = 0; i < NF / 8 * U; ++i) w[i] = a[i];
  }
  __device__ __forceinline__ void store_plain(T* row, int g) const {
    uint4* a = reinterpret_cast<uint4*>(row + NF * g);
#pragma unroll
    for (int i = 0; i < NF / 8 * U; ++i) a[i] = w[i];
  }
  __device__ __forceinline__ void turn(const Angles<D, MODE>& t, int g, int P) {
    float x[NF];
#pragma unroll
    for (int i = 0; i < NF / 8 * U; ++i) {
      const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
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
    float y[NF];
#pragma unroll
    for (int i = 0; i < NF / 2; ++i) {
      const int a = MODE == kAdjacent ? 2 * i : i, b = MODE == kAdjacent ? 2 * i + 1 : i + 8;
      const bool turns = MODE == kAdjacent ? 4 * g + i < P : 8 * g < P;
      y[a] = turns ? x[a] * t.c[i] - x[b] * t.s[i] : x[a];
      y[b] = turns ? x[a] * t.s[i] + x[b] * t.c[i] : x[b];
    }
#pragma unroll
    for (int i = 0; i < NF / 8 * U; ++i) {
      uint32_t v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 2) v[e] = pack_bf16(y[8 * i + 2 * e], y[8 * i + 2 * e + 1]);
        else v[e] = __float_as_uint(y[4 * i + e]);
      }
      w[i] = make_uint4(v[0], v[1], v[2], v[3]);
    }
  }
};

// rows from -> to (may be the same memory) of one token by thread g: the row of item i is from(i), to(i), for items i0 .. i1 - 1.
// A batch of rows is read before any of them is written: the compiler may not order them so, the memory may be the same.
template <typename T, int D, int MODE, class From, class To>
__device__ __forceinline__ void turn_rows(const Angles<D, MODE>& t, int g, int P, int i0, int i1, From from, To to) {
  if constexpr (MODE == kHalvesAny) {
    for (int i = i0; i < i1; ++i) {
      const T* x = from(i);
      T* y = to(i);
      float u[8], v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {   // slot p < P: features (p, p + P); the others follow behind 2 P
        const int p = 8 * g + e, a = p < P ? p : 2 * p, b = p < P ? p + P : 2 * p + 1;
        u[e] = Elem<T>::load(x + a);
        v[e] = Elem<T>::load(x + b);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int p = 8 * g + e, a = p < P ? p : 2 * p, b = p < P ? p + P : 2 * p + 1;
        Elem<T>::store(y + a, p < P ? u[e] * t.c[e] - v[e] * t.s[e] : u[e]);
        Elem<T>::store(y + b, p < P ? u[e] * t.s[e] + v[e] * t.c[e] : v[e]);
      }
    }
  } else {
    constexpr int U = 4;
    int i = i0;
    for (; i + U <= i1; i += U) {
      Piece16<T, D, MODE> p[U];
#pragma unroll
      for (int u = 0; u < U; ++u) p[u].load(from(i + u), g, P);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        p[u].turn(t, g, P);
        p[u].store(to(i + u), g, P);
      }
    }
    for (; i < i1; ++i) {
      Piece16<T, D, MODE> p;
      p.load(from(i), g, P);
      p.turn(t, g, P);
      p.store(to(i), g, P);
    }
  }
}

template <typename T, int D, int MODE, class From, class To>
__device__ __forceinline__ void copy_rows(int g, int i0, int i1, From from, To to) {
  constexpr int U = 4;
  int i = i0;
  for (; i + U <= i1; i += U) {
    Piece16<T, D, MODE> p[U];
#pragma unroll
    for (int u = 0; u < U; ++u) p[u].load_plain(from(i + u), g);
#pragma unroll
    for (int u = 0; u < U; ++u) p[u].store_plain(to(i + u), g);
  }
  for (; i < i1; ++i) {
    Piece16<T, D, MODE> p;
    p.load_plain(from(i), g);
    p.store_plain(to(i), g);
  }
}

// host.  A spectrum's rates are powers of one ratio, formed by products of 64 bits' precision: the 63rd is off by 2^-57 of itself, which
// a position of 2^31 makes a third of 2^-24 (a powl for each of 64 takes some microseconds of every call)
inline AxesSpec axes_spec(const hf_rope_axes& r) {
  AxesSpec s = {};
  s.n_axes = r.n_axes;
  for (int a = 0; a < r.n_axes; ++a) s.pairs += r.pairs[a];
  constexpr long double kTurn = 0.636619772367581343075535053490057448L;   // 2 / pi
  const auto ratio_of = [&](int n) { return powl((long double)r.theta, -1.0L / n); };
  long double quarter = kTurn, ratio = ratio_of(s.pairs);
  int p = 0;
  for (int a = 0; a < r.n_axes; ++a) {
    if (r.spectrum == HF_ROPE_PER_AXIS) {
      quarter = kTurn;
      ratio = ratio_of(r.pairs[a]);
    }
    for (int i = 0; i < r.pairs[a]; ++i, ++p) {
      s.quarter[p] = (double)quarter;
      s.rest[p] = (float)(quarter - s.quarter[p]);
      s.axis[p >> 4] |= (uint32_t)a << (2 * (p & 15));
      quarter *= ratio;
    }
  }
  return s;
}

inline AxesMode axes_mode(const hf_rope_axes& r, int pairs) {
  return r.layout == HF_ROPE_ADJACENT ? kAdjacent : pairs % 8 == 0 ? kHalves : kHalvesAny;
}

}  // namespace hf
