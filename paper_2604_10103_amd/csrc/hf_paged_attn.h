// Attention over a cache of pages: what its kernels share (internal).
//
// Rows.  The query heads of a group read the same keys, so a sequence's rows are numbered token by token, head by head of the group:
// row x of (sequence, key head h) is token x / group, query head h * group + x % group.  A workgroup takes BM of them.
//
// Items.  The grid is fixed by sizes that the host knows (packed rows, sequences, heads); which (sequence, rows, key head, part of the
// keys) a workgroup works on follows from the lengths, which only the device knows: every wavefront derives it for itself from cu_new
// and seq_lens, 64 sequences at a time, without exchange.  Keys count in tiles of 32.  A sequence whose rows see w tiles at most is cut
// into ceil(w / C) parts of equal length, C = ceil(longest w / S).  S is the one of 64 candidates (one a lane) for which a model of the
// launch is least: with n = the work in row tiles as long as the longest, x = n S / compute units,
//     rounds(x) * (longest w / S * tile + start) + (S > 1 ? meet + join * S : 0)      microseconds,
// rounds(x) = x rounded up where all rows see as much, else x + 3/4 (workgroups take what is next as they become free).  Only S with
// n S <= target are looked at (and S = 1), so that there are at most target + (row tiles) * heads_kv items, of which 2 * target are parts.
//
// Parts of a row meet in the workspace: each writes its sums (fp32) there, the last one to arrive adds them in the order of the parts.
#pragma once

#include <type_traits>

#include "hf_paged.h"

namespace hf {

constexpr int kKeyTile = 32;
constexpr float kComputeUnits = 256;

struct PagedSchedule {
  int target, capacity;          // capacity: parts that the workspace holds
  float tile, tile_alone;        // microseconds a tile takes where the chip is full, and at least
  float start, meet, join;
  unsigned long long* counters;  // [capacity] arrivals at a row tile, indexed by its first part
  float* parts;                  // [capacity][BM][D], behind them [capacity][BM][2]: row maximum and sum
  unsigned long long tag;
  bool by_xcd;                   // consecutive items on one XCD (they read the same keys)
};

struct PagedLaunch {   // the kernels' only argument
  PagedAttnArgs a;
  PagedSchedule sc;
};
// The arguments, read anew: kept over a kernel's phases they fill the scalar registers, and the loop would fetch spilled ones lane by lane
__device__ __forceinline__ PagedLaunch launch_arguments() {
  typedef const __attribute__((address_space(4))) uint32_t* Words;
  static_assert(sizeof(PagedLaunch) % 4 == 0, "words");
  Words p = (Words)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  struct { uint32_t w[sizeof(PagedLaunch) / 4]; } words;
#pragma unroll
  for (size_t i = 0; i < sizeof(PagedLaunch) / 4; ++i) words.w[i] = p[i];
  PagedLaunch r = __builtin_bit_cast(PagedLaunch, words);
  const auto global = [](auto& at) {   // (of an argument as such the compiler would know)
    at = (std::remove_reference_t<decltype(at)>)(__attribute__((address_space(1))) std::remove_pointer_t<std::remove_reference_t<decltype(at)>>*)reinterpret_cast<uintptr_t>(at);
  };
  global(r.a.Q); global(r.a.K_pages); global(r.a.V_pages); global(r.a.O); global(r.a.cu); global(r.a.lens); global(r.a.table); global(r.a.lse2);
  global(r.sc.counters); global(r.sc.parts);
  return r;
}

// the key tiles of some rows: 0 .. s1 - 1 (sink), then from s1 + skip on; n of them
struct KeyTiles {
  int s1, skip, n;
  __device__ __forceinline__ int start(int t) const { return kKeyTile * (t < s1 ? t : t + skip); }
};

// tokens t_lo .. t_hi of a sequence with m new tokens and `len` in all, of which `held` can lie in the cache
__device__ __forceinline__ KeyTiles key_tiles(const PagedAttnArgs& a, int m, int len, int held, int t_lo, int t_hi) {
  const int p_lo = len - m + t_lo, p_hi = len - m + t_hi;
  const int end = a.causal ? max(0, min(held, p_hi + 1)) : held;
  const int w1 = (end + kKeyTile - 1) / kKeyTile;
  KeyTiles k = {0, 0, w1};
  if (a.window > 0) {
    const int w0 = (int)(max(0ll, (long long)p_lo - a.window + 1) / kKeyTile);
    k.s1 = (min(a.n_sink, end) + kKeyTile - 1) / kKeyTile;
    k.skip = max(0, w0 - k.s1);
    k.n = min(k.s1, w1) + max(0, w1 - max(w0, k.s1));
  }
  return k;
}

struct PagedItem {
  int seq, begin, m, len, held;   // first packed row, new tokens, length, tokens that can lie in the cache
  int head_kv, first, rows;       // rows first .. first + rows - 1 of the sequence
  int part, parts, slot, counter; // which part of how many; its place in the workspace, and its row tile's counter
  int t0, t1;                     // its key tiles
  KeyTiles keys;
};

template <int BM> __device__ __forceinline__ bool find_item(const PagedAttnArgs& a, const PagedSchedule& sc, int item, PagedItem& it) {
  const int lane = threadIdx.x & 63, group = a.heads / a.heads_kv;
  const int most = a.max_pages * a.page;
  int begin = 0, m = 0, len = 0, T = 0, w = 0, w_least = 0;   // T row tiles that see w_least .. w key tiles
  auto look = [&](int s) {
    begin = m = len = T = w = w_least = 0;
    if (s < a.n_seqs) {
      begin = min(max(a.cu[s], 0), a.n_q);
      m = min(max(a.cu[s + 1], begin), a.n_q) - begin;
      len = max(a.lens[s], 0);
      if (m > 0) {
        T = (m * group + BM - 1) / BM;
        const int held = min(len, most);
        const KeyTiles x = key_tiles(a, m, len, held, 0, min(m, (BM - 1) / group + 1) - 1);
        const KeyTiles y = key_tiles(a, m, len, held, (T - 1) * BM / group, m - 1);
        w = max(1, max(x.n, y.n));
        w_least = max(1, min(x.n, y.n));
      }
    }
  };
  float most_units = 0.0f, units = 0.0f, rows = 0.0f, longest = 1.0f;
  for (int s0 = 0; s0 < a.n_seqs; s0 += kWave) {
    look(s0 + lane);
    most_units += (float)T * (float)w;
    units += (float)T * 0.5f * (float)(w + w_least);
    rows += (float)T;
    longest = fmaxf(longest, (float)w);
  }
  int C = 0x3fffffff;
  if (sc.capacity > 0) {
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      most_units += __shfl_xor(most_units, o, kWave);
      units += __shfl_xor(units, o, kWave);
      rows += __shfl_xor(rows, o, kWave);
      longest = fmaxf(longest, __shfl_xor(longest, o, kWave));
    }
    const float n = units / longest * (float)a.heads_kv;
    const float S = lane < 32 ? (float)(lane + 1) : floorf(32.0f * __builtin_amdgcn_exp2f((float)(lane - 31) * (5.0f / 32.0f)));   // .. 1024
    const float x = n * S * (1.0f / kComputeUnits);
    const float rounds = x <= 1.0f ? 1.0f : (units > 0.98f * longest * rows ? ceilf(x) : x + 0.75f);
    float cost = rounds * (longest / S * fmaxf(sc.tile_alone, sc.tile * fminf(x, 1.0f)) + sc.start) + (lane > 0 ? sc.meet + sc.join * S : 0.0f);
    if (lane > 0 && (most_units / longest * (float)a.heads_kv * S > (float)sc.target || S > longest)) cost = INFINITY;
    float best = cost;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) best = fminf(best, __shfl_xor(best, o, kWave));
    const int at = __ffsll(__ballot(cost == best)) - 1;
    const float s_best = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(S), at));
    if (at > 0) C = __builtin_amdgcn_readfirstlane((int)ceilf(longest / s_best));
  }
  // items of one key head: the item's head, and its place among them
  int each = 0, split_each = 0;
  for (int s0 = 0; s0 < a.n_seqs; s0 += kWave) {
    if (a.n_seqs > kWave) look(s0 + lane);
    const int S = (w + C - 1) / C;
    each += T * S;
    split_each += S > 1 ? T * S : 0;
  }
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    each += __shfl_xor(each, o, kWave);
    split_each += __shfl_xor(split_each, o, kWave);
  }
  each = __builtin_amdgcn_readfirstlane(each);
  split_each = __builtin_amdgcn_readfirstlane(split_each);
  if (sc.by_xcd) {   // workgroup ids go round the XCDs: each takes one contiguous eighth of the items
    const int per = (each * a.heads_kv + 7) / 8, slot = item >> 3;
    if (slot >= per) return false;
    item = (item & 7) * per + slot;
  }
  if (item >= each * a.heads_kv || split_each * a.heads_kv > sc.capacity) return false;   // (the latter cannot be, see above)
  it.head_kv = item / each;
  item -= it.head_kv * each;
  int before = 0, split_before = 0;   // items and parts of the sequences before
  for (int s0 = 0; s0 < a.n_seqs; s0 += kWave) {
    if (a.n_seqs > kWave) look(s0 + lane);
    const int S = (w + C - 1) / C, mine = T * S;
    int upto = mine, split_upto = S > 1 ? mine : 0;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int u = __shfl_up(upto, o, kWave), v = __shfl_up(split_upto, o, kWave);
      if (lane >= o) { upto += u; split_upto += v; }
    }
    const unsigned long long owner = __ballot(item >= before + upto - mine && item < before + upto);
    if (owner) {
      const int src = __ffsll(owner) - 1;
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, src); };
      it.seq = s0 + src;
      it.begin = of(begin);
      it.m = of(m);
      it.len = of(len);
      it.held = min(it.len, most);
      it.parts = of(S);
      const int tiles = of(T), own = of(mine), idx = item - (before + of(upto) - own);
      const int slot0 = it.head_kv * split_each + split_before + of(split_upto) - own;   // (meant where there are parts)
      // within a sequence: part, then rows, the last ones (which see most) first
      it.part = idx / tiles;
      const int back = idx - it.part * tiles, r = tiles - 1 - back;
      it.slot = slot0 + idx;
      it.counter = slot0 + back;
      it.first = r * BM;
      it.rows = min(BM, it.m * group - it.first);
      it.keys = key_tiles(a, it.m, it.len, it.held, it.first / group, (it.first + it.rows - 1) / group);
      it.t0 = (int)((long long)it.keys.n * it.part / it.parts);
      it.t1 = (int)((long long)it.keys.n * (it.part + 1) / it.parts);
      return true;
    }
    before += __builtin_amdgcn_readlane(upto, 63);
    split_before += __builtin_amdgcn_readlane(split_upto, 63);
  }
  return false;
}

// which keys a row sees: those below hi that are at least lo or below sink
struct RowView {
  int lo, hi, sink;
  __device__ __forceinline__ bool sees(int key) const { return key < hi && (key >= lo || key < sink); }
  // of the 32 keys from `start` on, a bit each
  __device__ __forceinline__ uint32_t sees_tile(int start) const { return below(hi - start) & (~below(lo - start) | below(sink - start)); }
  __device__ static __forceinline__ uint32_t below(int n) { return (uint32_t)((1ull << min(max(n, 0), 32)) - 1); }
};
__device__ __forceinline__ RowView row_view(const PagedAttnArgs& a, const PagedItem& it, int token) {
  const int p = it.len - it.m + token;
  RowView v;
  v.hi = a.causal ? max(0, min(it.held, p + 1)) : it.held;
  v.lo = a.window > 0 ? (int)max(0ll, (long long)p - a.window + 1) : 0;
  v.sink = a.window > 0 ? a.n_sink : 0;
  return v;
}

// ---- pages
typedef const __attribute__((address_space(4))) int32_t* ScalarInts;   // read through the scalar unit: a uniform address, not written meanwhile

__device__ __forceinline__ bool is_page(const PagedAttnArgs& a, int id) { return (unsigned)id < (unsigned)a.n_pages; }
__device__ __forceinline__ int div_page(const PagedAttnArgs& a, int key) {   // key / a.page for 0 <= key < 2^31
  return (int)(((unsigned long long)(unsigned)key * a.page_magic) >> a.page_shift);
}
// whether one of the item's entries is no page (uniform; every wavefront looks at all of them)
__device__ __forceinline__ bool any_bad_page(const PagedAttnArgs& a, const PagedItem& it) {
  if (it.t1 <= it.t0 || it.held == 0) return false;
  const int32_t* row = a.table + (long long)it.seq * a.max_pages;
  bool bad = false;
  auto scan = [&](int t0, int t1) {   // tiles t0 .. t1 - 1
    const int last = div_page(a, min(it.keys.start(t1 - 1) + kKeyTile, it.held) - 1);
    for (int e = div_page(a, it.keys.start(t0)) + (int)(threadIdx.x & 63); e <= last; e += kWave) bad = bad || !is_page(a, row[e]);
  };
  if (it.t0 < it.keys.s1) scan(it.t0, min(it.t1, it.keys.s1));
  if (it.t1 > it.keys.s1) scan(max(it.t0, it.keys.s1), it.t1);
  return __any(bad);
}

// x where bit k of `mask` is set, else -inf: without a condition register, of which sixteen at a time are too many
__device__ __forceinline__ float masked_score(float x, uint32_t mask, int k) {
  const uint32_t sel = (uint32_t)__builtin_amdgcn_sbfe((int)mask, k, 1);
  return __uint_as_float((__float_as_uint(x) & sel) | (0xff800000u & ~sel));
}

// a row that has seen keys, but only scores of -inf, carries this as its sum: nothing next to a part with a finite score, NaN alone
constexpr float kOnlyInfinite = -1.0f;

// ---- The end of an item.  The wavefronts' sums lie in LDS: group u's rows at rows_at(u) as [row][D + 4] floats, (maximum, sum) of its
// rows at stats_at(u).  NT threads; D / 8 of them share a row.  `flag`: an int in LDS that the rows do not cover.
template <typename T, int D, int BM, int KS, int NT, class RowsAt, class StatsAt>
__device__ __forceinline__ void finish_item(const PagedAttnArgs& a, const PagedSchedule& sc, const PagedItem& it, RowsAt rows_at, StatsAt stats_at,
                                            int* flag) {
  constexpr int TPR = D / 8, PER = NT / TPR, PASS = (BM + PER - 1) / PER;
  const int tid = threadIdx.x, f = 8 * (tid % TPR), r0 = tid / TPR, group = a.heads / a.heads_kv;
  typedef unsigned long long u64;
  __syncthreads();
  auto meet = [&](int row, float* acc, float& M, float& L) {   // the groups' parts of a row
    float mu[KS], lu[KS];
    M = -INFINITY;
#pragma unroll
    for (int u = 0; u < KS; ++u) {
      const float2 st = *reinterpret_cast<const float2*>(stats_at(u) + 2 * row);
      mu[u] = st.x;
      lu[u] = st.y;
      M = fmaxf(M, st.x);
    }
    const float use = M == -INFINITY ? 0.0f : M;
    L = 0.0f;
    bool only = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
#pragma unroll
    for (int u = 0; u < KS; ++u) {
      const float wgt = __builtin_amdgcn_exp2f(mu[u] - use);
      only = only || lu[u] == kOnlyInfinite;
      L += lu[u] == kOnlyInfinite ? 0.0f : lu[u] * wgt;
      const float* x = rows_at(u) + row * (D + 4) + f;
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        const float4 v = *reinterpret_cast<const float4*>(x + e);
        acc[e] += v.x * wgt; acc[e + 1] += v.y * wgt; acc[e + 2] += v.z * wgt; acc[e + 3] += v.w * wgt;
      }
    }
    if (only && M == -INFINITY && L == 0.0f) L = kOnlyInfinite;
  };
  auto write = [&](int row, const float* acc, float M, float L) {
    const int x = it.first + row, token = x / group, head = it.head_kv * group + (x - token * group);
    const bool none = M == -INFINITY && L == 0.0f;   // (a NaN anywhere makes L one)
    const float inv = none ? 0.0f : (L == kOnlyInfinite ? __builtin_nanf("") : 1.0f / L);
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = none ? 0.0f : acc[e] * inv;
    T* out = static_cast<T*>(a.O) + (long long)(it.begin + token) * a.ot + (long long)head * a.oh + f;
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<uint4*>(out) = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
    } else {
      *reinterpret_cast<float4*>(out) = make_float4(y[0], y[1], y[2], y[3]);
      *reinterpret_cast<float4*>(out + 4) = make_float4(y[4], y[5], y[6], y[7]);
    }
    if (a.lse2 && f == 0)
      a.lse2[(long long)head * a.n_q + it.begin + token] = none ? INFINITY : (L == kOnlyInfinite ? __builtin_nanf("") : M + log2f(L));
  };
  if (it.parts == 1) {
#pragma unroll 1
    for (int p = 0; p < PASS; ++p) {
      const int row = r0 + p * PER;
      if (row >= it.rows) break;
      float acc[8], M, L;
      meet(row, acc, M, L);
      write(row, acc, M, L);
    }
    return;
  }
  // ---- a part: its sums go past the caches of this XCD (sc1), each store acknowledged before the arrival
  constexpr int kSc1 = 16;
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const __amdgpu_buffer_rsrc_t parts = __builtin_amdgcn_make_buffer_rsrc(sc.parts, 0, sc.capacity * (BM * (D + 2) * 4), 0x00020000);
  const int stats_at_byte = sc.capacity * (BM * D * 4);
  auto row_byte = [&](int slot, int row) { return (slot * BM + row) * (D * 4) + 4 * f; };
  auto stat_byte = [&](int slot, int row) { return stats_at_byte + (slot * BM + row) * 8; };
  u64* const counter = sc.counters + it.counter;
  if (tid == 0) {   // a counter of another call counts from zero
    u64 seen = __hip_atomic_load(counter, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if ((seen >> 16) != sc.tag)
      (void)__hip_atomic_compare_exchange_strong(counter, &seen, sc.tag << 16, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
#pragma unroll 1
  for (int p = 0; p < PASS; ++p) {
    const int row = r0 + p * PER;
    if (row >= it.rows) break;
    float acc[8], M, L;
    meet(row, acc, M, L);
    const int to = row_byte(it.slot, row);
    __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(acc[0]), __float_as_uint(acc[1]), __float_as_uint(acc[2]), __float_as_uint(acc[3])}, parts, to, 0, kSc1);
    __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(acc[4]), __float_as_uint(acc[5]), __float_as_uint(acc[6]), __float_as_uint(acc[7])}, parts, to + 16, 0, kSc1);
    if (f == 0) __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(M), __float_as_uint(L)}, parts, stat_byte(it.slot, row), 0, kSc1);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) {
    const u64 before = __hip_atomic_fetch_add(counter, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const int last = (int)(before & 0xffffu) == it.parts - 1;
    if (last) __hip_atomic_store(counter, sc.tag << 16, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // ready for a replay
    *flag = last;
  }
  __syncthreads();
  if (!*flag) return;
  // ---- the last one.  The parts of (row tile, key head) lie as many slots apart as the sequence has row tiles.  Few rows leave threads
  // over: G sets of threads then take every G-th part each and meet in LDS, in their order
  const int tiles = (it.m * group + BM - 1) / BM;
  int lanes_rows = 1;                                   // rows of a pass, a power of two
  while (lanes_rows < it.rows && lanes_rows < PER) lanes_rows *= 2;
  const int G = PER / lanes_rows, set = r0 / lanes_rows, rp = r0 % lanes_rows;
  constexpr int LINE = 8 * TPR + 4;                     // floats of a row in LDS: sums, then (maximum, sum)
  float* const meeting = const_cast<float*>(rows_at(0));
  const int passes = (it.rows + lanes_rows - 1) / lanes_rows;
  // R rows (of passes p ..) times U parts are requested together: few parts of many rows, or many parts of few
  auto join = [&](auto r_of, auto u_of, int p, float (&M)[decltype(r_of)::value], float (&L)[decltype(r_of)::value], float (&acc)[decltype(r_of)::value][8]) {
    constexpr int R = decltype(r_of)::value, U = decltype(u_of)::value;
    bool only[R];
    int row[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      M[r] = -INFINITY;
      L[r] = 0.0f;
      only[r] = false;
      row[r] = min(rp + (p + r) * lanes_rows, it.rows - 1);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[r][e] = 0.0f;
    }
#pragma unroll 1
    for (int u0 = set; u0 < it.parts; u0 += U * G) {
      u32x2 st[R][U];
      u32x4 v[R][U][2];
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const int slot = it.counter + min(u0 + i * G, it.parts - 1) * tiles;
          st[r][i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(parts, stat_byte(slot, row[r]), 0, kSc1));
          v[r][i][0] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(parts, row_byte(slot, row[r]), 0, kSc1));
          v[r][i][1] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(parts, row_byte(slot, row[r]) + 16, 0, kSc1));
        }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float top = M[r];
#pragma unroll
        for (int i = 0; i < U; ++i) top = fmaxf(top, u0 + i * G < it.parts ? __uint_as_float(st[r][i][0]) : -INFINITY);
        const float use = top == -INFINITY ? 0.0f : top, w0 = __builtin_amdgcn_exp2f(M[r] - use);
        M[r] = top;
        L[r] *= w0;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[r][e] *= w0;
#pragma unroll
        for (int i = 0; i < U; ++i) {
          if (u0 + i * G >= it.parts) break;
          const float wgt = __builtin_amdgcn_exp2f(__uint_as_float(st[r][i][0]) - use), l = __uint_as_float(st[r][i][1]);
          only[r] = only[r] || l == kOnlyInfinite;
          L[r] += l == kOnlyInfinite ? 0.0f : l * wgt;
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[r][e] += __uint_as_float(v[r][i][e >> 2][e & 3]) * wgt;
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (only[r] && M[r] == -INFINITY && L[r] == 0.0f) L[r] = kOnlyInfinite;
  };
  if (G == 1) {
    auto all_rows = [&](auto r_of, auto u_of) {
      constexpr int R = decltype(r_of)::value;
#pragma unroll 1
      for (int p = 0; p < passes; p += R) {
        float M[R], L[R], acc[R][8];
        join(r_of, u_of, p, M, L, acc);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const int row = rp + (p + r) * lanes_rows;
          if (row < it.rows) write(row, acc[r], M[r], L[r]);
        }
      }
    };
    if (it.parts <= 2) all_rows(std::integral_constant<int, 4>{}, std::integral_constant<int, 2>{});
    else if (it.parts <= 4) all_rows(std::integral_constant<int, 2>{}, std::integral_constant<int, 4>{});
    else all_rows(std::integral_constant<int, 1>{}, std::integral_constant<int, 8>{});
    return;
  }
  float Ms[1], Ls[1], sum[1][8];
  join(std::integral_constant<int, 1>{}, std::integral_constant<int, 8>{}, 0, Ms, Ls, sum);
  float* const line = meeting + r0 * LINE;
#pragma unroll
  for (int e = 0; e < 8; e += 4) *reinterpret_cast<float4*>(line + f + e) = make_float4(sum[0][e], sum[0][e + 1], sum[0][e + 2], sum[0][e + 3]);
  if (f == 0) *reinterpret_cast<float2*>(line + 8 * TPR) = make_float2(Ms[0], Ls[0]);
  __syncthreads();
  if (set != 0 || rp >= it.rows) return;
  const float* from = meeting + rp * LINE;
  float M = -INFINITY, L = 0.0f, acc[8];
  for (int g = 0; g < G; ++g) M = fmaxf(M, from[g * lanes_rows * LINE + 8 * TPR]);
  const float use = M == -INFINITY ? 0.0f : M;
  bool only = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
  for (int g = 0; g < G; ++g) {
    const float* x = from + g * lanes_rows * LINE;
    const float l = x[8 * TPR + 1], wgt = __builtin_amdgcn_exp2f(x[8 * TPR] - use);
    only = only || l == kOnlyInfinite;
    L += l == kOnlyInfinite ? 0.0f : l * wgt;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += x[f + e] * wgt;
  }
  if (only && M == -INFINITY && L == 0.0f) L = kOnlyInfinite;
  write(rp, acc, M, L);
}

}  // namespace hf
