// Attention over a cache of pages in 8 bits (hf_paged_attn_e4m3_fwd): bf16 or fp32 queries, head_dim 64 or 128.
//
// A code of e4m3 is a bf16 with three of its seven mantissa bits in use, so that codes are converted without loss (one instruction for two)
// and multiplied on the bf16 matrix cores as they are.  A key's scale is a factor of its scores, a value's of its probability:
//     s_j = c ks_j (q . kc_j),   o = sum_j (p_j vs_j) vc_j / sum_j p_j,
// both in fp32.  fp32 queries and the products p vs are split into three bf16 each (8 + 8 + 8 bits: nothing is lost), whose products
// accumulate in fp32.  In bf16 the products p vs are two bf16 where rows are few: 16 bits, and outputs as far off 64 bits as exact products
// leave them, 1.66e-3, their own rounding (rounded to one bf16 2.34e-3).  That kernel waits for memory: 64 single tokens over 410 to 8191 keys
// take 116.7 us, with one 115.8; 16 drafts of 8 tokens 48.9 and 48.2.  In chunks they are rounded to one (half a step of each, which averages
// out over the keys: 2.3e-3), as there the second half costs a third: 12 heads x 4680 over 9360 to 14040 keys 624 us, with one 468.
//
// Both products are transposed, S^T = K Q^T and O^T += V^T P^T, so that a lane holds scores of one row and the exponentials are the second
// product's operand as they lie.  Rows, work, parts and the end of an item are those of the other paged kernels (hf_paged_attn.h).
//
// Two kernels:
//   few rows (16 or 32 a workgroup: single tokens)   bound by memory: 64 single tokens over 410 to 8191 keys 117 us, 5.1 TB/s.  Every wavefront
//                                                    reads its own tiles as bytes, global -> LDS directly, and converts what it has read into registers
//   chunks (128 or 256 rows a workgroup)             bound by the vector unit beside the matrix cores: 12 heads x 4680 over 9360 to 14040 keys
//                                                    467 us, 800 TFLOP/s.  K is converted once on its way into LDS, where all wavefronts read it as bf16
#include "hf_e4m3.h"
#include "hf_paged_attn.h"

namespace hf {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

namespace {

struct E4m3Launch {   // the kernels' only argument; launch_arguments() reads the first part anew
  PagedLaunch paged;
  const float *k_scales, *v_scales;
};

// 8 codes as bf16
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi) {
  const u32x4 w = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true))};
  return __builtin_bit_cast(bf16x8, w);
}

// the codes of four that are NaN: their bytes' top bits
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// NaN where bit k of `bad` is set and the row sees the key, else 0, to be added: by arithmetic (an assignment under the condition came out of
// the compiler, clang 22, with the sums lost in the rows that the condition spares)
__device__ __forceinline__ float nan_where(uint32_t bad, int k, bool sees) {
  return __uint_as_float((bad >> k & (uint32_t)sees & 1u) * 0x7fc00000u);
}

// PL bf16 whose sum is x (three: all of fp32's bits; one: rounded)
template <int PL> __device__ __forceinline__ void split(float x, __bf16 (&p)[PL]) {
#pragma unroll
  for (int i = 0; i < PL; ++i) {
    p[i] = static_cast<__bf16>(x);
    x -= static_cast<float>(p[i]);
  }
}
// 8 consecutive elements of a row
template <typename T, int PL> __device__ __forceinline__ void load_planes(const T* from, bf16x8 (&p)[PL]) {
  if constexpr (sizeof(T) == 2) {
    p[0] = *reinterpret_cast<const bf16x8*>(from);
  } else {
    float x[8];
    load16B(from, x);
    load16B(from + 4, x + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      __bf16 s[PL];
      split(x[e], s);
#pragma unroll
      for (int i = 0; i < PL; ++i) p[i][e] = s[i];
    }
  }
}

__device__ __forceinline__ uint32_t and_mask(float x, uint32_t mask, int k) {   // x where bit k of `mask` is set, else 0
  return __float_as_uint(x) & (uint32_t)__builtin_amdgcn_sbfe((int)mask, k, 1);
}

constexpr int kNoKeys = 0x60000000;   // where a tile that there is not would start: behind every sequence (2^30), and no sum with it overflows

// where the keys of an item's tiles lie: the pool's row (0 where there is none: read, and masked).  The wavefront keeps 64 entries of the
// table, from ids_base on, a lane each.  Tiles start at multiples of 32
struct PoolRows {
  const int32_t* table;
  uint32_t page_rows, head_rows;
  int ids, ids_base, key_last, entry_last;
  int two_at = -(1 << 30), two_inside = 0;
  uint32_t two_rows = 0;
  __device__ __forceinline__ PoolRows(const PagedAttnArgs& a, const PagedItem& it)
      : table(a.table + (long long)it.seq * a.max_pages), page_rows((uint32_t)a.heads_kv * (uint32_t)a.page),
        head_rows((uint32_t)it.head_kv * (uint32_t)a.page), ids(-1), ids_base(-kWave), key_last(it.held - 1),
        entry_last(it.held > 0 ? div_page(a, it.held - 1) : 0) {}
  // of the keys of two tiles, at s0 and s1 (>= held: none), lane by lane, where the last call's were 64 keys before: a page that holds both has
  // its rows 64 further (of keys behind the sequence's the page's own, if there is one)
  __device__ __forceinline__ uint32_t next_two(const PagedAttnArgs& a, int s0, int s1, int lane, bool bad_pages) {
    const bool follows = s0 - 2 * kKeyTile == two_at && s1 == s0 + kKeyTile && s0 <= key_last && !bad_pages;   // (uniform)
    two_at = s0;
    if (follows && two_inside + 2 * kKeyTile + 63 < a.page) {   // (the first key's place; uniform)
      two_inside += 2 * kKeyTile;
      return two_rows += 2 * kKeyTile;
    }
    two_inside = s0 <= key_last ? s0 - div_page(a, s0) * a.page : a.page;
    return two_rows = rows(a, s0, s1, lane);
  }
  // the same, found anew
  __device__ __forceinline__ uint32_t rows(const PagedAttnArgs& a, int s0, int s1, int lane) {
    if (s1 == s0 + kKeyTile) return run<2 * kKeyTile>(a, s0, lane);   // (uniform)
    const uint32_t r0 = run<kKeyTile>(a, s0, lane & 31), r1 = run<kKeyTile>(a, s1, lane & 31);
    return lane < 32 ? r0 : r1;
  }
  __device__ __forceinline__ uint32_t row(const PagedAttnArgs& a, int start, int lane) { return run<kKeyTile>(a, start, lane & 31); }
  // of N <= 64 keys from `start` on: of key start + at
  template <int N> __device__ __forceinline__ uint32_t run(const PagedAttnArgs& a, int start, int at) {
    if (start > key_last) return 0;   // (uniform)
    const int first = div_page(a, start), last = div_page(a, min(start + N - 1, key_last));
    if (first < ids_base || last >= ids_base + kWave) {
      const int lane = thread_id() & 63;
      ids_base = first;
      ids = first + lane <= entry_last ? table[first + lane] : -1;
      // waited for here: where the paths join, the compiler would wait for these in every call, and so for all other requests
      __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
    }
    const int key = min(start + at, key_last), entry = div_page(a, key);
    int id;
    if (last <= first + 1) {   // two pages at most: no exchange through LDS, which would be waited for
      const int id0 = __builtin_amdgcn_readlane(ids, first - ids_base), id1 = __builtin_amdgcn_readlane(ids, last - ids_base);
      id = entry == first ? id0 : id1;
    } else {
      id = __shfl(ids, entry - ids_base, kWave);
    }
    return is_page(a, id) ? (uint32_t)id * page_rows + head_rows + (uint32_t)(key - entry * a.page) : 0;
  }
};

// the tiles of which rows from `lo`'s view to `hi`'s see all keys (uniform): first .. first + n - 1 of the wavefront's, `base` its first one
struct FullTiles {
  int first, n;
  __device__ __forceinline__ FullTiles(const PagedAttnArgs& a, const PagedItem& it, int base, const RowView& lo, const RowView& hi, bool bad) {
    const auto index_of = [&](int tile) { return max(0, max(it.keys.s1, tile - it.keys.skip) - base); };
    first = index_of(tiles_to(a, hi.lo));
    n = bad ? 0 : max(0, index_of(tile_of(a, lo.hi)) - first);
  }
  __device__ __forceinline__ bool has(int i) const { return (unsigned)(i - first) < (unsigned)n; }
};

// NaN codes next to rows that do not see them were left out: they enter the sums of the rows that do.  Off the fast path, key by key, straight
// from the pages: add(key, the pool's row) for each key that exists, of the tiles that some row sees in part
template <class Start, class Full, class F>
__device__ __forceinline__ void each_key(const PagedAttnArgs& a, const PagedItem& it, const PoolRows& rows, int count, Start start_of, Full full, F add) {
#pragma unroll 1
  for (int i = 0; i < count; ++i) {
    if (full(i)) continue;
    const int start = start_of(i);
#pragma unroll 1
    for (int key = start; key < min(start + kKeyTile, it.held); ++key) {
      const int entry = div_page(a, key), id = rows.table[entry];
      if (is_page(a, id)) add(key, (uint64_t)((uint32_t)id * rows.page_rows + rows.head_rows + (uint32_t)(key - entry * a.page)));
    }
  }
}

// ------------------------------------------------------------------------------------------------ few rows
// RB blocks of 16 rows a workgroup, KS wavefronts that share the keys, a run of tiles each, and meet at the end.  Products are 16 x 16 x 32
// (features or keys): lane (n, g) = (lane % 16, lane / 16).  S^T: row n of the block, keys 16 t + 4 g + r.  A lane's features of K and Q are
// D / 4 consecutive ones, eight a step (which order the sum takes does not matter as long as both take it).  V^T: feature 16 dt + n, keys
// 4 g .. + 3 and 16 + 4 g .. + 3, by reads that transpose 8 keys x 16 features of bytes.
// Two tiles of codes and scales (8.25 KB each at head_dim 128) are on their way or at work: with eight wavefronts a compute unit 132 KB.
template <int D, int RB, int KS> struct FewShape {
  static constexpr int BM = 16 * RB, NT = 64 * KS;
  static constexpr int TILE = kKeyTile * D, SLOT = 2 * TILE + 256;   // codes of K, of V, scales of both
  static constexpr int OUT = BM * (D + 4) * 4 + BM * 8;
  static constexpr int SPAN = (2 * SLOT > OUT ? 2 * SLOT : OUT) + 255 & ~255;
  static constexpr int LDS = KS * SPAN + 16;                         // (an int behind all)
};

// 16-byte unit u of row r sits at u ^ swizzle(r): the lanes that are served together find all banks
template <int D> __device__ __forceinline__ int k8_swizzle(int r) { return D == 128 ? (r >> 1) & 7 : (r >> 2) & 3; }
template <int D> __device__ __forceinline__ int v8_swizzle(int r) {
  return D == 128 ? ((r >> 1) & 3) | ((r >> 4) & 1) << 2 : ((r >> 2) & 1) | ((r >> 4) & 1) << 1;
}

template <typename T, int D, int RB, int KS>
__global__ __launch_bounds__(64 * KS, sizeof(T) == 2 ? 2 : 1) void e4m3_few_kernel(const E4m3Launch args) {
  using S = FewShape<D, RB, KS>;
  constexpr int BM = S::BM, TILE = S::TILE, SLOT = S::SLOT, PL = sizeof(T) == 2 ? 1 : 3;
  constexpr int PP = sizeof(T) == 2 ? 2 : 3;               // bf16 of a product p vs (PL: of a query's element)
  constexpr int NS = D / 32, ND = D / 16;                  // steps of S^T, blocks of 16 features of O^T
  constexpr int RPP = 1024 / D, UPR = D / 16, NP = kKeyTile / RPP;   // rows of a 1 KB piece, 16-byte units of a row, pieces of a tile
  constexpr int REQ = 2 * NP + 1;                          // requests of a tile
  extern __shared__ __attribute__((aligned(256))) char smem[];

  PagedCursor cursor;
  {
    const PagedLaunch p = launch_arguments();
    cursor = first_item<BM, true, true>(p.a, p.sc);
  }
  for (bool again = false;; again = true) {
  PagedItem it;
  {
    const PagedLaunch p = launch_arguments();
    if (!next_item<BM, true>(p.a, p.sc, cursor, it)) return;
  }
  if (again) __syncthreads();   // everybody is done with the sums in LDS
  const PagedAttnArgs a = launch_arguments().a;

  const int tid = thread_id(), lane = tid & 63, n = lane & 15, g = lane >> 4, group = a.group;
  const int grp = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6);
  char* const base = smem + grp * S::SPAN;

  // ---- this lane's rows (past the item's rows: its last one again; only the rows that there are get stored)
  const int x_last = it.first + it.rows - 1;
  RowView view[RB];
  bf16x8 qf[RB][NS][PL];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int x = min(it.first + 16 * rb + n, x_last), token = div_group(a, x);
    view[rb] = row_view(a, it, token);
    const T* q = static_cast<const T*>(a.Q) + (long long)(it.begin + token) * a.qt + (long long)(it.head_kv * group + (x - token * group)) * a.qh +
                 D / 4 * g;
#pragma unroll
    for (int s = 0; s < NS; ++s) load_planes<T, PL>(q + 8 * s, qf[rb][s]);
  }
  const bool bad_pages = any_bad_page(a, it);

  // ---- the wavefront's tiles
  const int run = (it.t1 - it.t0 + KS - 1) / KS, base_tile = it.t0 + grp * run, count = max(0, min(run, it.t1 - base_tile));
  const auto start_of = [&](int i) { return i < count ? kKeyTile * it.keys.tile(base_tile + i) : kNoKeys; };
  const FullTiles full(a, it, base_tile, row_view(a, it, div_group(a, it.first)), row_view(a, it, div_group(a, x_last)), bad_pages);

  // ---- requests: a tile's 1 KB pieces, lane's row of piece j: RPP j + lane / UPR; and its scales, a lane each (K's, then V's)
  PoolRows pool(a, it);
  const uint64_t k_pool = reinterpret_cast<uint64_t>(a.K_pages), v_pool = reinterpret_cast<uint64_t>(a.V_pages);
  const uint64_t s_pool = reinterpret_cast<uint64_t>(lane < 32 ? args.k_scales : args.v_scales);
  typedef __attribute__((address_space(3))) char* Lds;
  const uint32_t lds = (uint32_t)(uintptr_t)(Lds)base;
  const auto to_lds_16 = [](uint32_t dst, uint64_t from) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :: "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(from) : "memory", "m0");
  };
  const auto to_lds_4 = [](uint32_t dst, uint64_t from) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                 :: "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(from) : "memory", "m0");
  };
  const auto request = [&](uint32_t rows, uint32_t slot) {
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int r = RPP * j + lane / UPR, u = lane % UPR;
      const uint64_t row = (uint64_t)(uint32_t)__shfl((int)rows, r, kWave) * D;
      to_lds_16(slot + 1024 * j, k_pool + row + 16 * (u ^ k8_swizzle<D>(r)));
      to_lds_16(slot + TILE + 1024 * j, v_pool + row + 16 * (u ^ v8_swizzle<D>(r)));
    }
    to_lds_4(slot + 2 * TILE, s_pool + 4 * (uint64_t)rows);
  };

  // ---- LDS reads, within a slot
  const int k_at = n * D, ks = k8_swizzle<D>(n);           // (the swizzles of rows 16 apart agree)
  const int v_row = (lane & 8 ? 16 : 0) + 4 * g + ((lane >> 1) & 3);
  const uint32_t v_at = lds + TILE + v_row * D + 16 * v8_swizzle<D>(v_row) + 8 * (lane & 1);

  f32x4 o[RB][ND];
  float m_ref[RB], l_run[RB];
  uint32_t seen[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[rb][dt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    m_ref[rb] = -INFINITY;
    l_run[rb] = 0.0f;
    seen[rb] = 0;
  }
  bool odd = false;   // NaN codes lie next to rows that do not see them: they were left out (uniform)

  // the rows have to be here before the first request: the compiler does not count requests, and a wait behind them would be one for all
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int pl = 0; pl < PL; ++pl) asm volatile("" : "+v"(qf[rb][s][pl]));
  if (count > 0) {
    const uint32_t row0 = pool.row(a, start_of(0), lane), row1 = pool.row(a, start_of(1), lane);
    request(row0, lds);
    request(row1, lds + SLOT);
  }
  uint32_t row_next = count > 0 ? pool.row(a, start_of(2), lane) : 0;

#pragma unroll 1
  for (int i = 0; i < count; ++i) {
    const uint32_t slot = (i & 1) * SLOT;
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(REQ) : "memory");   // tile i; the next one may fly
    u32x4 kr[2][D / 64];
    i32x2 vr[ND];
    f32x4 ksc[2], vsc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int u = 0; u < D / 64; ++u) kr[t][u] = *reinterpret_cast<const u32x4*>(base + slot + k_at + 16 * t * D + 16 * ((D / 64 * g + u) ^ ks));
      ksc[t] = *reinterpret_cast<const f32x4*>(base + slot + 2 * TILE + 64 * t + 16 * g);
      vsc[t] = *reinterpret_cast<const f32x4*>(base + slot + 2 * TILE + 128 + 64 * t + 16 * g);
    }
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
      vr[dt] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((i32x2 __attribute__((address_space(3)))*)(uintptr_t)((v_at + slot) ^ (16 * dt)));
    const uint32_t rows = row_next;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the slot has been read
    request(rows, lds + slot);
    row_next = pool.row(a, start_of(i + 3), lane);

    // ---- S^T
    f32x4 s[RB][2];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int t = 0; t < 2; ++t) s[rb][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int st = 0; st < NS; ++st)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bf16x8 kf = widen(kr[t][st / 2][2 * (st & 1)], kr[t][st / 2][2 * (st & 1) + 1]);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int pl = PL - 1; pl >= 0; --pl) s[rb][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[rb][st][pl], s[rb][t], 0, 0, 0);
      }
    const bool all = full.has(i);
    uint32_t existing = 0xffffffffu;
    if (!all) {
      const int start = start_of(i);
      if (bad_pages) {
        const int key = start + (lane & 31);
        existing = (uint32_t)__ballot(key < it.held && is_page(a, pool.table[div_page(a, min(key, it.held - 1))]));
      }
      // a probability of zero does not make a NaN vanish: such codes become zero here
      uint32_t any = 0;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) any |= nan_codes((uint32_t)vr[dt][0]) | nan_codes((uint32_t)vr[dt][1]);
      if (__any(any != 0)) {
        odd = true;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
          for (int e = 0; e < 2; ++e) vr[dt][e] = (int)((uint32_t)vr[dt][e] & ~((nan_codes((uint32_t)vr[dt][e]) >> 7) * 255u));
      }
    }
    bf16x8 pf[RB][PP];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = s[rb][e >> 2][e & 3] * (ksc[e >> 2][e & 3] * a.c_scale);
      uint32_t mine = 0;
      if (!all) {
        const uint32_t sees = view[rb].sees_tile(start_of(i)) & existing;
        seen[rb] |= sees;
        mine = sees >> (4 * g);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = masked_score(x[e], mine, 16 * (e >> 2) + (e & 3));
      } else {
        seen[rb] = 1;
      }
      // ---- online softmax in the exp2 domain (a row with a NaN keeps its reference: its sum is NaN in any case)
      float mx = max_of3(max_of3(x[0], x[1], x[2]), max_of3(x[3], x[4], x[5]), max_of3(x[6], x[7], x[7]));
      {
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        mx = max_of3(__uint_as_float(sw[0]), __uint_as_float(sw[1]), __uint_as_float(sw[1]));
        const auto sv = __builtin_amdgcn_permlane16_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        mx = max_of3(__uint_as_float(sv[0]), __uint_as_float(sv[1]), __uint_as_float(sv[1]));
      }
      const bool grows = mx > m_ref[rb] + kGrow;
      if (__any(grows)) {
        const float m_new = grows ? mx : m_ref[rb];
        const float alpha = grows ? __builtin_amdgcn_exp2f(m_ref[rb] - m_new) : 1.0f;
        m_ref[rb] = m_new;
        l_run[rb] *= alpha;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) o[rb][dt] *= alpha;
      }
      const float m_use = m_ref[rb] == -INFINITY ? 0.0f : m_ref[rb];
      float psum = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p = __builtin_amdgcn_exp2f(x[e] - m_use);
        psum += p;
        x[e] = p * vsc[e >> 2][e & 3];
      }
      l_run[rb] += psum;
      if (!all) {   // (a scale that is not finite)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(and_mask(x[e], mine, 16 * (e >> 2) + (e & 3)));
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        __bf16 p[PP];
        split(x[e], p);
#pragma unroll
        for (int pl = 0; pl < PP; ++pl) pf[rb][pl][e] = p[pl];
      }
    }
    // ---- O^T += V^T P^T
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) {
      const bf16x8 vf = widen((uint32_t)vr[dt][0], (uint32_t)vr[dt][1]);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int pl = PP - 1; pl >= 0; --pl) o[rb][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[rb][pl], o[rb][dt], 0, 0, 0);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing may land on the sums

  if (odd)
    each_key(a, it, pool, count, start_of, [&](int i) { return full.has(i); }, [&](int key, uint64_t row) {
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) {
        const uint32_t bad = nan_codes(*(const __attribute__((address_space(1))) uint32_t*)(v_pool + row * D + 16 * dt + 4 * g));
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[rb][dt][r] += nan_where(bad, 8 * r + 7, view[rb].sees(key));
      }
    });

  // ---- the sums of the wavefront's rows go to LDS
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run[rb]), __float_as_uint(l_run[rb]), false, false);
    float l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    const auto sv = __builtin_amdgcn_permlane16_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(sv[0]) + __uint_as_float(sv[1]);
    if (seen[rb] != 0 && m_ref[rb] == -INFINITY && l == 0.0f) l = kOnlyInfinite;
    float* const row = reinterpret_cast<float*>(base) + (16 * rb + n) * (D + 4);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) *reinterpret_cast<f32x4*>(row + 16 * dt + 4 * g) = o[rb][dt];
    if (g == 0) *reinterpret_cast<float2*>(reinterpret_cast<float*>(base) + BM * (D + 4) + 2 * (16 * rb + n)) = make_float2(m_ref[rb], l);
  }
  const PagedLaunch p = launch_arguments();
  finish_item<T, D, BM, KS, S::NT>(
      p.a, p.sc, it, [&](int u) { return reinterpret_cast<const float*>(smem + u * S::SPAN); },
      [&](int u) { return reinterpret_cast<const float*>(smem + u * S::SPAN) + BM * (D + 4); }, reinterpret_cast<int*>(smem + KS * S::SPAN));
  }
}

template <int D> __device__ __forceinline__ int v8_swizzle_32(int r) {   // where the lanes that are served together read 16 features of 8 keys each
  return D == 128 ? ((r >> 1) & 1) << 1 | ((r >> 3) & 1) << 2 : ((r >> 3) & 1) << 1;
}

// ------------------------------------------------------------------------------------------------ chunks
// NW wavefronts of 32 rows each share every tile of 32 keys.  Products are 32 x 32 x 16, as in the other paged kernel: lane (l32, h) holds
// row l32's scores of the keys 8 j + 4 h + r.  K goes through registers and into LDS as bf16, with the scales beside it (a key's times c); V
// goes there directly, as bytes, which every wavefront converts behind its transposing reads: of bf16 those would take the LDS twice as long.
// Two tiles lie in a slot, one barrier for both, and what brings the next ones runs under a product.  Steps of that, 12 heads x 4680 over 9360
// to 14040 keys: both converted on the way, a barrier a tile 558 us; two tiles a barrier and V as bytes 513; the way under the first product, a
// page's rows by addition 482; wavefronts without rows in a loop of their own, no order of instructions given 467.
template <int D, int NW> struct ChunkShape {
  static constexpr int BM = 32 * NW, NT = 64 * NW;
  static constexpr int ROWB = 2 * D, KT = kKeyTile * ROWB, VT = kKeyTile * D;    // a tile of K as bf16, of V as bytes
  static constexpr int V = 6 * KT, SCALES = V + 6 * VT;                          // three slots of two tiles each; of scales, two
  static constexpr int OUT = BM * (D + 4) * 4 + BM * 8;
  static constexpr int SPAN = SCALES + 1024 > OUT ? SCALES + 1024 : OUT;
  static constexpr int LDS = SPAN + 16;
};

template <typename T, int D, int NW>
__global__ __launch_bounds__(64 * NW, sizeof(T) == 2 ? 2 : 1) void e4m3_chunk_kernel(const E4m3Launch args) {
  using S = ChunkShape<D, NW>;
  constexpr int BM = S::BM, NT = S::NT, ROWB = S::ROWB, KT = S::KT, VT = S::VT, PL = sizeof(T) == 2 ? 1 : 3;
  constexpr int NS = D / 16, ND = D / 32;                  // steps of S^T, 32-feature blocks of O^T
  constexpr int TPR = NT / (2 * kKeyTile), CPT = D / TPR;  // threads of a key's row, and their codes
  static_assert(CPT == 16 || CPT == 32, "16 bytes, once or twice");
  extern __shared__ __attribute__((aligned(256))) char smem[];

  PagedItem it;
  {
    const PagedLaunch p = launch_arguments();
    PagedCursor cursor = first_item<BM, false>(p.a, p.sc);
    if (!next_item<BM, false>(p.a, p.sc, cursor, it)) return;
  }
  const PagedAttnArgs a = launch_arguments().a;
  const int tid = thread_id(), lane = tid & 63, l32 = lane & 31, h = lane >> 5, group = a.group;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // ---- this lane's row (past the item's rows: its last one again; only the rows that there are get stored)
  const int x_last = it.first + it.rows - 1, x = min(it.first + 32 * wave + l32, x_last), token = div_group(a, x);
  const RowView view = row_view(a, it, token);
  const bool active = 32 * wave < it.rows;                 // (uniform)
  bf16x8 qf[NS][PL];
  {
    const T* q = static_cast<const T*>(a.Q) + (long long)(it.begin + token) * a.qt + (long long)(it.head_kv * group + (x - token * group)) * a.qh +
                 8 * h;
#pragma unroll
    for (int s = 0; s < NS; ++s) load_planes<T, PL>(q + 16 * s, qf[s]);
  }
  const bool bad_pages = any_bad_page(a, it);
  const int count = max(0, it.t1 - it.t0);
  const auto start_of = [&](int i) { return i < count ? kKeyTile * it.keys.tile(it.t0 + i) : kNoKeys; };
  const FullTiles full(a, it, it.t0, row_view(a, it, div_group(a, min(it.first + 32 * wave, x_last))),
                       row_view(a, it, div_group(a, min(it.first + 32 * wave + 31, x_last))), bad_pages);

  // ---- the way of two tiles into LDS.  The wavefront knows their rows, a lane each
  PoolRows pool(a, it);
  typedef __attribute__((address_space(3))) char* Lds;
  const uint32_t lds = (uint32_t)(uintptr_t)(Lds)smem;
  // K and the scales through registers: this thread's key, and its codes of it
  const int key_in = tid / TPR, part = tid % TPR;
  const uint8_t* const k_from = static_cast<const uint8_t*>(a.K_pages) + CPT * part;
  struct Codes {
    u32x4 w[CPT / 16];
  };
  const auto fetch_k = [&](uint32_t row) {
    Codes c;
#pragma unroll
    for (int u = 0; u < CPT / 16; ++u) c.w[u] = reinterpret_cast<const u32x4*>(k_from + (uint64_t)row * D)[u];
    return c;
  };
  struct Scales {
    float k, v;
  };
  const auto fetch_scales = [&](uint32_t row) { return Scales{args.k_scales[row], args.v_scales[row]}; };
  const auto place_k = [&](const Codes& c, int slot) {
    char* const to = smem + 2 * KT * slot + key_in * ROWB;   // (a tile's rows are those of the next one's)
#pragma unroll
    for (int u = 0; u < CPT / 8; ++u)
      *reinterpret_cast<bf16x8*>(to + 16 * ((CPT / 8 * part + u) ^ k_swizzle<D>(key_in & 31))) = widen(c.w[u / 2][2 * (u & 1)], c.w[u / 2][2 * (u & 1) + 1]);
  };
  const auto place_scales = [&](const Scales& sc, int slot) {
    float* const to = reinterpret_cast<float*>(smem + S::SCALES + 512 * slot) + key_in;
    if (part == 0) {
      to[0] = sc.k * a.c_scale;
      to[64] = sc.v;
    }
  };
  // V as it is: 1 KB pieces, a wavefront's are NW apart
  constexpr int RPP = 1024 / D, UPR = D / 16, NP = 2 * VT / 1024 / NW;   // keys of a piece, 16-byte units of a key, a wavefront's pieces
  static_assert(NP == 1 || NP == 2, "pieces");
  const uint64_t v_pool = reinterpret_cast<uint64_t>(a.V_pages);
  struct VRows {
    uint32_t r[NP];
  };
  const auto bring_v = [&](const VRows& rows, int slot) {
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int key = (RPP * (wave + NW * j) + lane / UPR) & 31;
      const uint64_t from = v_pool + (uint64_t)rows.r[j] * D + 16 * ((lane % UPR) ^ v8_swizzle_32<D>(key));
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                   :: "s"(__builtin_amdgcn_readfirstlane(lds + S::V + 2 * VT * slot + 1024 * (wave + NW * j))), "v"(from) : "memory", "m0");
    }
  };

  // ---- LDS reads.  K fragment of step s: unit 2 s + h of row l32.  V^T fragment (feature 32 dt + l32; keys 16 t2 + 8 y + 4 h .. + 3) by
  // transposing reads: a 16-lane group fetches 8 keys x 16 features in chunks of 8 bytes
  uint32_t k_addr[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) k_addr[s] = lds + l32 * ROWB + 16 * ((2 * s + h) ^ k_swizzle<D>(l32));
  const int v_row = 4 * h + ((lane >> 1) & 3) + (lane & 8);   // (the swizzles of rows 16 apart agree)
  const uint32_t v_at = lds + S::V + v_row * D + 16 * (((lane >> 4) & 1) ^ v8_swizzle_32<D>(v_row)) + 8 * (lane & 1);

  f32x16 o[ND];
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.0f;
  float m_ref = -INFINITY, l_run = 0.0f;
  uint32_t seen = 0;

  bool odd = false;   // NaN codes lie next to rows that do not see them: they were left out (uniform)

  bf16x8 kf[NS];
  const auto read_k = [&](int slot) {
#pragma unroll
    for (int s = 0; s < NS; ++s) kf[s] = *(const __attribute__((address_space(3))) bf16x8*)(uintptr_t)(k_addr[s] + slot * KT);
  };
  Codes kc;    // on their way: when step p begins, K of the tiles of step p + 1, their scales' and V's of p (V into LDS)
  Scales sc;
  uint32_t row_k = 0, row_s = 0;   // the thread's rows of what is requested next
  VRows row_v = {};
  uint32_t rows_next = 0;          // the wavefront's, of the step's tiles behind those
  const auto k_row_of = [&](uint32_t rows) { return (uint32_t)__shfl((int)rows, key_in, kWave); };
  const auto v_rows_of = [&](uint32_t rows) {
    VRows v;
#pragma unroll
    for (int j = 0; j < NP; ++j) v.r[j] = (uint32_t)__shfl((int)rows, RPP * (wave + NW * j) + lane / UPR, kWave);
    return v;
  };

  // step p's share of this, into `slot`
  const auto on_the_way = [&](int p, const int slot) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0): what the last step has requested, V included
    place_k(kc, slot);
    place_scales(sc, p & 1);
    bring_v(row_v, slot);
    kc = fetch_k(row_k);
    sc = fetch_scales(row_s);
    row_s = row_k;
    row_v = v_rows_of(rows_next);
    rows_next = pool.next_two(a, start_of(2 * p + 6), start_of(2 * p + 7), lane, bad_pages);
    row_k = k_row_of(rows_next);
  };

  // tile i, the first or second (half) of the two in a slot, whose K fragments are in registers.  Behind the first one's product, and the next
  // tiles' way while it runs, everybody meets: K of the next slot and V of this one are there, and nobody is at the slot before any more
  const auto tile = [&](int i, const int slot, const int half) __attribute__((always_inline)) {
    const int par = (i / 2) & 1;
    f32x16 sacc;
#pragma unroll
    for (int r = 0; r < 16; ++r) sacc[r] = 0.0f;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int pl = PL - 1; pl >= 0; --pl) sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s], qf[s][pl], sacc, 0, 0, 0);
    if (half == 0) {
      if (i > 0) on_the_way(i / 2, (slot + 1) % 3);
      __syncthreads();
    }
    // what the softmax needs first, then what the products need
    const uint32_t scales = lds + S::SCALES + 512 * par + 128 * half + 16 * h;
    const int v_off = VT * (2 * slot + half);
    const auto four = [&](int j) { return *(const __attribute__((address_space(3))) f32x4*)(uintptr_t)(scales + 16 * j); };
    f32x4 ks[4], vs[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) ks[j] = four(2 * j);
    i32x2 vr[2][ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2)
        vr[t2][dt] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((i32x2 __attribute__((address_space(3)))*)(uintptr_t)((v_at ^ (32 * dt)) + v_off + 16 * D * t2));
    read_k(half == 0 ? 2 * slot + 1 : (2 * slot + 2) % 6);
    const float m_use = m_ref == -INFINITY ? 0.0f : m_ref;   // exponents against the row's reference, which rarely moves
#pragma unroll
    for (int r = 0; r < 16; ++r) sacc[r] = fmaf(sacc[r], ks[r >> 2][r & 3], -m_use);
    const bool all = full.has(i);
    uint32_t mine = 0;
    if (!all) {
      const int start = start_of(i);
      uint32_t existing = 0xffffffffu;
      if (bad_pages) {
        const int key = start + l32;
        existing = (uint32_t)__ballot(key < it.held && is_page(a, pool.table[div_page(a, min(key, it.held - 1))]));
      }
      const uint32_t sees = view.sees_tile(start) & existing;
      mine = sees >> (4 * h);
      seen |= sees;
#pragma unroll
      for (int r = 0; r < 16; ++r) sacc[r] = masked_score(sacc[r], mine, 8 * (r >> 2) + (r & 3));
      // a probability of zero does not make a NaN vanish: such codes become zero here
      uint32_t any = 0;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2) any |= nan_codes((uint32_t)vr[t2][dt][0]) | nan_codes((uint32_t)vr[t2][dt][1]);
      if (__any(any != 0)) {
        odd = true;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
          for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              vr[t2][dt][e] = (int)((uint32_t)vr[t2][dt][e] & ~((nan_codes((uint32_t)vr[t2][dt][e]) >> 7) * 255u));
      }
    } else {
      seen = 1;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) vs[j] = four(16 + 2 * j);
    // ---- online softmax in the exp2 domain (a row with a NaN keeps its reference: its sum is NaN in any case)
    float mx = max_of3(max_of3(max_of3(sacc[0], sacc[1], sacc[2]), max_of3(sacc[3], sacc[4], sacc[5]), max_of3(sacc[6], sacc[7], sacc[8])),
                       max_of3(sacc[9], sacc[10], sacc[11]), max_of3(sacc[12], sacc[13], max_of3(sacc[14], sacc[15], sacc[15])));
    {
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = max_of3(__uint_as_float(sw[0]), __uint_as_float(sw[1]), __uint_as_float(sw[1]));
    }
    const bool grows = mx > (m_ref == -INFINITY ? -INFINITY : kGrow);
    if (__any(grows)) {
      const float more = grows ? mx : 0.0f, m_new = grows ? m_use + mx : m_ref;
      const float alpha = grows ? __builtin_amdgcn_exp2f(m_ref - m_new) : 1.0f;
      m_ref = m_new;
      l_run *= alpha;
#pragma unroll
      for (int r = 0; r < 16; ++r) sacc[r] -= more;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
    }
    float psum = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      sacc[r] = __builtin_amdgcn_exp2f(sacc[r]);
      psum += sacc[r];
    }
    l_run += psum;
#pragma unroll
    for (int r = 0; r < 16; ++r) sacc[r] *= vs[r >> 2][r & 3];
    if (!all) {   // (a scale that is not finite)
#pragma unroll
      for (int r = 0; r < 16; ++r) sacc[r] = __uint_as_float(and_mask(sacc[r], mine, 8 * (r >> 2) + (r & 3)));
    }
    bf16x8 pf[2][PL];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      __bf16 p[PL];
      split(sacc[r], p);
#pragma unroll
      for (int pl = 0; pl < PL; ++pl) pf[r >> 3][pl][r & 7] = p[pl];
    }
    // ---- O^T += V^T P^T
#pragma unroll
    for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) {
        const bf16x8 vf = widen((uint32_t)vr[t2][dt][0], (uint32_t)vr[t2][dt][1]);
#pragma unroll
        for (int pl = PL - 1; pl >= 0; --pl) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[t2][pl], o[dt], 0, 0, 0);
      }
  };
  const auto step = [&](int p, const int slot) __attribute__((always_inline)) {
    tile(2 * p, slot, 0);
    if (2 * p + 1 < count) tile(2 * p + 1, slot, 1);
  };

  if (count > 0) {
    const uint32_t r0 = pool.rows(a, start_of(0), start_of(1), lane), r1 = pool.rows(a, start_of(2), start_of(3), lane);
    const uint32_t r2 = pool.rows(a, start_of(4), start_of(5), lane);
    const Codes k0 = fetch_k(k_row_of(r0)), k1 = fetch_k(k_row_of(r1));
    const Scales s0 = fetch_scales(k_row_of(r0));
    bring_v(v_rows_of(r0), 0);
    bring_v(v_rows_of(r1), 1);
    row_s = k_row_of(r2);
    kc = fetch_k(row_s);
    sc = fetch_scales(k_row_of(r1));
    row_v = v_rows_of(r2);
    rows_next = pool.next_two(a, start_of(6), start_of(7), lane, bad_pages);
    row_k = k_row_of(rows_next);
    place_k(k0, 0);
    place_scales(s0, 0);
    place_k(k1, 1);
  }
  // nothing is on its way any more.  (Else the compiler would wait for the queries where the loop uses them, and so in every step for what that
  // step has requested itself)
  __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
  __syncthreads();
  if (active) {
    if (count > 0) read_k(0);
#pragma unroll 1
    for (int p = 0; 2 * p < count; p += 3) {
      step(p, 0);
      if (2 * p + 2 >= count) break;
      step(p + 1, 1);
      if (2 * p + 4 >= count) break;
      step(p + 2, 2);
    }
  } else {   // no rows: the wavefront only carries its share of the tiles
    int slot = 1;
#pragma unroll 1
    for (int p = 0; 2 * p < count; ++p) {
      if (p > 0) {
        slot = slot == 2 ? 0 : slot + 1;
        on_the_way(p, slot);
      }
      __syncthreads();
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing may land on the sums
  __syncthreads();   // the sums lie over the tiles

  if (odd)
    each_key(a, it, pool, count, start_of, [&](int i) { return full.has(i); }, [&](int key, uint64_t row) {
      const uint64_t v_pool = reinterpret_cast<uint64_t>(a.V_pages);
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t bad = nan_codes(*(const __attribute__((address_space(1))) uint32_t*)(v_pool + row * D + 32 * dt + 8 * q + 4 * h));
#pragma unroll
          for (int r = 0; r < 4; ++r) o[dt][4 * q + r] += nan_where(bad, 8 * r + 7, view.sees(key));
        }
    });

  // ---- the sums of the wavefront's rows go to LDS
  {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
    l_run = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    if (seen != 0 && m_ref == -INFINITY && l_run == 0.0f) l_run = kOnlyInfinite;
    float* const row = reinterpret_cast<float*>(smem) + (32 * wave + l32) * (D + 4);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(row + 32 * dt + 8 * q + 4 * h) = make_float4(o[dt][4 * q], o[dt][4 * q + 1], o[dt][4 * q + 2], o[dt][4 * q + 3]);
    if (h == 0) *reinterpret_cast<float2*>(reinterpret_cast<float*>(smem) + BM * (D + 4) + 2 * (32 * wave + l32)) = make_float2(m_ref, l_run);
  }
  const PagedLaunch p = launch_arguments();
  finish_item<T, D, BM, 1, NT>(
      p.a, p.sc, it, [&](int) { return reinterpret_cast<const float*>(smem); },
      [&](int) { return reinterpret_cast<const float*>(smem) + BM * (D + 4); }, reinterpret_cast<int*>(smem + S::SPAN));
}

// ---- launches
struct Plan {
  int rows, grid, ks;   // rows of a workgroup, groups that share their keys
  PagedSchedule sc;
};

Plan plan_of(const hf_paged& c, int n_q) {
  const int group = c.heads / c.heads_kv;
  const long long rows = (long long)n_q * group;
  Plan p = {};
  auto tiles = [&](int of) { return (rows / of + (n_q < c.n_seqs ? n_q : c.n_seqs)) * c.heads_kv; };   // row tiles of all heads, at most
  // what a sequence has on the average: up to 16 rows, up to 32, or chunks
  p.rows = rows <= 16ll * c.n_seqs ? 16 : rows <= 32ll * c.n_seqs ? 32 : 128;
  if (p.rows == 128 && c.dtype == HF_BF16 && c.head_dim == 128 && rows > 128ll * c.n_seqs) {
    const long long n = (rows + c.n_seqs - 1) / c.n_seqs, heads = (long long)c.n_seqs * c.heads_kv;   // (as if all were as long)
    auto rounds = [&](int of) { return (double)(((n + of - 1) / of * heads + 255) / 256); };
    // (microseconds a tile of two earlier kernels; the schedule below has 0.89 and 0.535, a ratio of 1.66 for 1.85.  12 heads x 4680 over 9360 to
    // 14040 keys take 470 us by 256 rows, 516 by 128; 16 heads x 8 x 512 over 2012 85 and 90.  Where lengths differ the rule, which does not know
    // them, errs: 8 sequences of up to 512 new over up to 1500 take 82 by 256 rows, which it chooses, and 71 by 128)
    if (rounds(256) * 1.10 <= rounds(128) * 0.595) p.rows = 256;
  }
  p.ks = p.rows <= 32 ? 4 : 1;
  const bool wide = c.head_dim == 128;
  const long long key_tiles = ((long long)c.max_pages * c.page_tokens + kKeyTile - 1) / kKeyTile;   // (at most)
  if (p.rows <= 32) {
    // Eight wavefronts share a row tile's keys, one workgroup a compute unit, where there are few row tiles or their keys may be many: half as
    // many parts of a row meet (four tokens over 131071 keys 65 us, with four wavefronts and two workgroups a unit 84; 64 single tokens over 410 to
    // 8191 117 and 134; 8 over 800 to 16000 36 and 42; eight tokens over 60000 44 and 65).  More row tiles of shorter sequences find two to four
    // chains on their unit, each of which waits for its own: 64 single tokens over 1025 keys 34 us by eight wavefronts, 28 by four; 200 over 100 to
    // 2000 119 and 105; and, where there is one for all 2048 wavefronts, a row tile a wavefront.
    if (tiles(p.rows) >= 2048) {
      p.ks = 1;
      p.sc.groups = kMostGroups;
      p.sc.tile = wide ? 3.2f : 1.6f;
      p.sc.tile_alone = wide ? 1.2f : 0.9f;
      p.sc.lead = 2;
    } else if ((c.dtype == HF_BF16 || p.rows == 16) && (tiles(p.rows) <= 400 || key_tiles >= 112)) {
      p.ks = 8;
      p.sc.groups = 256;
      p.sc.tile = wide ? 0.4f : 0.2f;
      p.sc.tile_alone = wide ? 0.3f : 0.2f;
      p.sc.lead = 10;
    } else {
      p.sc.groups = 512;
      p.sc.tile = wide ? 0.8f : 0.4f;
      p.sc.tile_alone = wide ? 0.3f : 0.2f;
      p.sc.lead = 5;
    }
    p.sc.units = (float)p.sc.groups;
    p.sc.start = 4.0f;
    p.sc.meet = 5.0f;
    p.sc.join = 0.1f;
  } else {
    p.sc.units = 256.0f;            // (two or three workgroups that run on a unit at a time share its products)
    p.sc.groups = 65536 / p.rows;   // (at most 512)
    p.sc.meet = 6.0f;
    p.sc.join = 1.0f;
    p.sc.start = 5.0f;
    if (c.dtype == HF_F32) {
      p.sc.tile = wide ? 2.0f : 1.2f;
      p.sc.tile_alone = wide ? 2.2f : 1.4f;
      p.sc.start = 9.0f;
    } else if (p.rows == 256) {
      p.sc.tile = p.sc.tile_alone = 0.89f;
      p.sc.start = 9.0f;
    } else {
      p.sc.tile = wide ? 0.535f : 0.29f;
      p.sc.tile_alone = wide ? 0.7f : 0.4f;
    }
  }
  long long grid = p.rows <= 32 ? p.sc.groups : tiles(p.rows) + p.sc.groups;
  if (grid > tiles(p.rows) * key_tiles) grid = tiles(p.rows) * key_tiles;
  p.grid = (int)((grid + 7) & ~7ll);
  p.sc.meets = key_tiles > 1;
  return p;
}

template <auto* Kernel, class S> int launch(const E4m3Launch& l, int grid, hipStream_t s) {
  static LdsGrant grant;
  const int rc = grant_lds(grant, reinterpret_cast<const void*>(Kernel), S::LDS, "hf_paged_attn_e4m3_fwd");
  if (rc != HF_OK) return rc;
  hipLaunchKernelGGL(Kernel, dim3(grid), dim3(S::NT), S::LDS, s, l);
  return check_launch("hf_paged_attn_e4m3_fwd");
}

template <typename T, int D> int launch_of(const E4m3Launch& l, const Plan& p, hipStream_t s) {
  if constexpr (D == 128 && sizeof(T) == 2) {
    if (p.rows == 256) return launch<e4m3_chunk_kernel<T, D, 8>, ChunkShape<D, 8>>(l, p.grid, s);
  }
  if (p.rows == 128) return launch<e4m3_chunk_kernel<T, D, 4>, ChunkShape<D, 4>>(l, p.grid, s);
  if (p.rows == 32) {
    if constexpr (sizeof(T) == 2) {   // (fp32: more registers than eight wavefronts have)
      if (p.ks == 8) return launch<e4m3_few_kernel<T, D, 2, 8>, FewShape<D, 2, 8>>(l, p.grid, s);
    }
    if (p.ks == 1) return launch<e4m3_few_kernel<T, D, 2, 1>, FewShape<D, 2, 1>>(l, p.grid, s);
    return launch<e4m3_few_kernel<T, D, 2, 4>, FewShape<D, 2, 4>>(l, p.grid, s);
  }
  if (p.ks == 8) return launch<e4m3_few_kernel<T, D, 1, 8>, FewShape<D, 1, 8>>(l, p.grid, s);
  if (p.ks == 1) return launch<e4m3_few_kernel<T, D, 1, 1>, FewShape<D, 1, 1>>(l, p.grid, s);
  return launch<e4m3_few_kernel<T, D, 1, 4>, FewShape<D, 1, 4>>(l, p.grid, s);
}

}  // namespace

long long paged_e4m3_threads(const hf_paged& c, int n_q) {
  const Plan p = plan_of(c, n_q);
  return (long long)p.grid * (p.rows <= 32 ? 64 * p.ks : 2 * p.rows);
}

size_t paged_e4m3_workspace_bytes(const hf_paged& c, int n_q) {
  if (n_q == 0) return 0;
  const Plan p = plan_of(c, n_q);
  if (!p.sc.meets) return 0;
  return kCounterBytes + (size_t)p.sc.groups * 2 * p.rows * (c.head_dim + 2) * 4;
}

int launch_paged_attn_e4m3(const hf_paged& c, PagedAttnArgs a, const float* K_scales, const float* V_scales, void* workspace, hipStream_t s) {
  const Plan p = plan_of(c, a.n_q);
  a.page_shift = magic_of(c.page_tokens, a.page_magic);
  a.group = c.heads / c.heads_kv;
  a.group_shift = magic_of(a.group, a.group_magic);
  PagedSchedule sc = p.sc;
  if (sc.meets) {
    sc.counters = static_cast<unsigned long long*>(workspace);
    sc.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + kCounterBytes);
    sc.tag = next_call_tag();
  }
  const E4m3Launch l = {{a, sc}, K_scales, V_scales};
  if (c.dtype == HF_BF16) return c.head_dim == 128 ? launch_of<bf16_t, 128>(l, p, s) : launch_of<bf16_t, 64>(l, p, s);
  return c.head_dim == 128 ? launch_of<float, 128>(l, p, s) : launch_of<float, 64>(l, p, s);
}

}  // namespace hf
