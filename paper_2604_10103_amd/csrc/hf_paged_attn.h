// Attention over a cache of pages: what its kernels share (internal).
//
// Rows.  The query heads of a group read the same keys, so a sequence's rows are numbered token by token, head by head of the group:
// row x of (sequence, key head h) is token x / group, query head h * group + x % group.  A workgroup takes BM of them.
//
// Items.  The grid is fixed by sizes that the host knows (packed rows, sequences, heads); which (sequence, rows, key head, part of the
// keys) a workgroup works on follows from the lengths, which only the device knows: every wavefront derives it for itself from cu_new
// and seq_lens, 64 sequences at a time, without exchange.  Keys count in tiles of 32.  A sequence whose rows see w tiles at most is cut
// into S = ceil(w / C) parts of equal length, C = max(cmin, all tiles of all rows / target): about `target` parts of like size in all,
// whatever the lengths are.  There are at most target + (row tiles) * heads_kv items, and at most 2 * target that are parts.
//
// Parts of a row meet in the workspace: each writes its sums (fp32) there, the last one to arrive adds them in the order of the parts.
#pragma once

#include "hf_paged.h"

namespace hf {

constexpr int kKeyTile = 32;

struct PagedSchedule {
  int target, cmin, capacity;    // parts that the workspace holds
  unsigned long long* counters;  // [capacity] arrivals at a row tile, indexed by its first part
  float* parts;                  // [capacity][BM][D], behind them [capacity][BM][2]: row maximum and sum
  unsigned long long tag;
  bool by_xcd;                   // consecutive items on one XCD (they read the same keys)
};

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
  int begin = 0, m = 0, len = 0, T = 0, w = 0;
  auto look = [&](int s) {
    begin = m = len = T = w = 0;
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
      }
    }
  };
  float units = 0.0f;
  for (int s0 = 0; s0 < a.n_seqs; s0 += kWave) {
    look(s0 + lane);
    units += (float)T * (float)w;
  }
  units = wave_sum(units);
  const int C = max(sc.cmin, (int)ceilf(fminf(units * (float)a.heads_kv / (float)sc.target, 1e9f)));
  if (sc.by_xcd) {   // workgroup ids go round the XCDs: each takes one contiguous eighth of the items
    int total = 0;
    for (int s0 = 0; s0 < a.n_seqs; s0 += kWave) {
      if (a.n_seqs > kWave) look(s0 + lane);
      total += T * ((w + C - 1) / C) * a.heads_kv;
    }
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) total += __shfl_xor(total, o, kWave);
    const int per = (total + 7) / 8, slot = item >> 3;
    if (slot >= per) return false;
    item = (item & 7) * per + slot;
  }
  int before = 0, split_before = 0;   // items and parts of the sequences before
  for (int s0 = 0; s0 < a.n_seqs; s0 += kWave) {
    if (a.n_seqs > kWave) look(s0 + lane);
    const int S = (w + C - 1) / C, mine = T * S * a.heads_kv;
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
      const int slot0 = split_before + of(split_upto) - own;   // (meant where there are parts)
      // within a sequence: key head, part, then rows, the last ones (which see most) first
      const int x = idx / tiles, r = tiles - 1 - (idx - x * tiles);
      it.head_kv = x / it.parts;
      it.part = x - it.head_kv * it.parts;
      it.slot = slot0 + idx;
      it.counter = slot0 + it.head_kv * it.parts * tiles + idx - x * tiles;
      if (it.parts > 1 && slot0 + own > sc.capacity) return false;   // (cannot be, see above)
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
  float* const part_rows = sc.parts;
  float* const part_stats = sc.parts + (size_t)sc.capacity * BM * D;
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
  // ---- a part: its sums go past the caches of this XCD, each store acknowledged before the arrival
  auto store2 = [](float* p, float x, float y) {
    __hip_atomic_store(reinterpret_cast<u64*>(p), (u64)__float_as_uint(x) | ((u64)__float_as_uint(y) << 32), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };
  auto load2 = [](const float* p) {
    const u64 v = __hip_atomic_load(const_cast<u64*>(reinterpret_cast<const u64*>(p)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
  };
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
    float* to = part_rows + ((size_t)it.slot * BM + row) * D + f;
#pragma unroll
    for (int e = 0; e < 8; e += 2) store2(to + e, acc[e], acc[e + 1]);
    if (f == 0) store2(part_stats + ((size_t)it.slot * BM + row) * 2, M, L);
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
  // ---- the last one: the parts of (row tile, key head) lie as many slots apart as the sequence has row tiles
  const int tiles = (it.m * group + BM - 1) / BM;
#pragma unroll 1
  for (int p = 0; p < PASS; ++p) {
    const int row = r0 + p * PER;
    if (row >= it.rows) break;
    float M = -INFINITY;
    const float* st = part_stats + ((size_t)it.counter * BM + row) * 2;
    const size_t st_step = (size_t)tiles * BM * 2;
#pragma unroll 8
    for (int u = 0; u < it.parts; ++u) M = fmaxf(M, load2(st + u * st_step).x);
    const float use = M == -INFINITY ? 0.0f : M;
    float L = 0.0f, acc[8];
    bool only = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
    const float* from = part_rows + ((size_t)it.counter * BM + row) * D + f;
#pragma unroll 4
    for (int u = 0; u < it.parts; ++u) {
      const float2 s = load2(st + u * st_step);
      const float wgt = __builtin_amdgcn_exp2f(s.x - use);
      only = only || s.y == kOnlyInfinite;
      L += s.y == kOnlyInfinite ? 0.0f : s.y * wgt;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float2 v = load2(from + (size_t)u * tiles * BM * D + e);
        acc[e] += v.x * wgt;
        acc[e + 1] += v.y * wgt;
      }
    }
    if (only && M == -INFINITY && L == 0.0f) L = kOnlyInfinite;
    write(row, acc, M, L);
  }
}

}  // namespace hf
