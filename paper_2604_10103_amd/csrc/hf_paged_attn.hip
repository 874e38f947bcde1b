// Attention over a cache of pages on bf16 MFMA (hf_paged_attn_fwd, bf16 storage, head_dim 64 or 128).
//
// The layout of the window kernels (hf_attn_mfma.hip): a wavefront owns 32 rows, tiles of 32 keys, both products transposed,
//   S^T (keys x rows) = K_tile (A, from LDS) x Q^T (B, registers),   O^T (d x rows) += V_tile^T (A, LDS) x P^T (B, registers),
// so that the statistics of a row are private to its two lanes and the exponentials of S^T are, rounded to bf16, the B operand of the
// second product.  K and V tiles go global -> LDS directly, V^T fragments are transposing reads, three K slots and two V slots.
// Here the rows are tokens x heads of a group, and a tile's 1 KB pieces (4 or 8 keys) each have a page of their own: their descriptors
// are scalar arithmetic on the entries of the page table, which a wavefront keeps 64 of, a lane each.  Pages of an odd number of tokens
// (page_tokens no multiple of a piece's keys) take an address per lane instead.
//
// Two shapes of workgroup (NW wavefronts of rows, KS groups of wavefronts that share the keys):
//   NW 4, KS 1   128 rows, tiles shared by four wavefronts, one barrier a tile: chunks, bound by the matrix cores and the softmax
//   NW 1, KS 4   32 rows, every wavefront its own tiles and no barrier until the end: single tokens, bound by memory
#include "hf_paged_attn.h"

namespace hf {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

namespace {

constexpr float kGrow = 8.0f;   // log2 units: a row's reference moves only when its maximum grew by more than 2^8

__device__ uint4 zero_row[1];   // what keys that are none read as, where a lane has an address

// 16-byte unit u of key row r sits at u ^ swizzle(r) (conflict-free fragment reads)
template <int D> __device__ __forceinline__ int k_swizzle(int r) {
  return D == 128 ? (r & 15) : (((r >> 1) & 1) | (((r >> 2) ^ (r >> 3)) & 1) << 1 | (((r >> 3) ^ (r >> 4)) & 1) << 2);
}
template <int D> __device__ __forceinline__ int v_swizzle(int r) {
  return D == 128 ? ((r & 3) << 2 | ((r >> 2) & 3)) : (((r >> 1) & 1) << 2 | ((r >> 2) & 3));
}

// max without the quieting of NaNs around fmaxf: a NaN score makes its row's sum one in any case
__device__ __forceinline__ float max3f(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

template <int D, int NW, int KS> struct Shape {
  static constexpr int BM = 32 * NW, NT = 64 * NW * KS;
  static constexpr int ROWB = 2 * D, TILE = kKeyTile * ROWB;
  static constexpr int KSLOTS = NW == 4 ? 4 : 3;
  static constexpr int GROUP = (KSLOTS + 2) * TILE;                  // a group's tiles: those of K, two of V
  static constexpr int OUT = BM * (D + 4) * 4 + BM * 8;              // a group's sums behind the loop, and its rows' statistics
  static constexpr int SPAN = GROUP > OUT ? GROUP : OUT;
  static constexpr int FLAG = GROUP > OUT ? OUT : KS * SPAN;         // an int behind the sums
  static constexpr int LDS = KS * SPAN + (GROUP > OUT ? 0 : 16);
};

// kWhole: a piece of a tile lies in one page (page_tokens a multiple of its keys)
template <int D, int NW, int KS, bool kWhole>
__global__ __launch_bounds__(64 * NW * KS, (NW == 4 ? 2 : 1)) void paged_attn_kernel(const PagedAttnArgs a, const PagedSchedule sc) {
  static_assert(NW == 1 || KS == 1, "groups share no barrier");
  using S = Shape<D, NW, KS>;
  constexpr int BM = S::BM, ROWB = S::ROWB, TILE = S::TILE, KSLOTS = S::KSLOTS;
  constexpr int RPP = 1024 / ROWB, UPR = ROWB / 16;       // keys of a 1 KB piece, 16-byte units of a key
  constexpr int CPT = kKeyTile / RPP / NW;                // pieces of a tile that a wavefront requests
  constexpr int NS = D / 16, ND = D / 32;                 // steps of S^T, 32-feature blocks of O^T
  extern __shared__ __attribute__((aligned(16))) char smem[];

  PagedItem it;
  if (!find_item<BM>(a, sc, blockIdx.x, it)) return;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave_in_wg = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave = KS == 1 ? wave_in_wg : 0, grp = KS == 1 ? 0 : wave_in_wg;
  char* const sK = smem + grp * S::SPAN;
  char* const sV = sK + KSLOTS * TILE;
  const int l32 = lane & 31, h = lane >> 5, group = a.heads / a.heads_kv;

  // ---- this lane's row (past the item's rows: its last one again; only the rows that there are get stored)
  const int x_last = it.first + it.rows - 1, x = min(it.first + 32 * wave + l32, x_last), token = x / group;
  const RowView view = row_view(a, it, token);
  const bool active = 32 * wave < it.rows;                 // (uniform)
  // what all rows of the wavefront see, and what any of them sees
  const RowView view_lo = row_view(a, it, min(it.first + 32 * wave, x_last) / group);
  const RowView view_hi = row_view(a, it, min(it.first + 32 * wave + 31, x_last) / group);
  bf16x8 qf[NS];
  {
    const bf16_t* q = static_cast<const bf16_t*>(a.Q) + (long long)(it.begin + token) * a.qt +
                      (long long)(it.head_kv * group + (x - token * group)) * a.qh + 8 * h;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(q + 16 * s);
  }
  const bool bad_pages = any_bad_page(a, it);

  // ---- the item's tiles t0 + grp, + KS, ... (every wavefront of a group the same)
  const int count = max(0, (it.t1 - it.t0 - grp + KS - 1) / KS);
  constexpr int kNone = 0x7fffffe0;                        // where no tile starts
  auto start_of = [&](int i) { return __builtin_amdgcn_readfirstlane(i < count ? it.keys.start(it.t0 + grp + KS * i) : kNone); };

  // ---- requests: piece j of this wavefront is the tile's keys RPP (wave + NW j) ..
  const uint64_t page_bytes = (uint64_t)a.heads_kv * (uint32_t)a.page * ROWB, head_bytes = (uint64_t)it.head_kv * (uint32_t)a.page * ROWB;
  const uint64_t k_pool = reinterpret_cast<uint64_t>(a.K_pages) + head_bytes, v_pool = reinterpret_cast<uint64_t>(a.V_pages) + head_bytes;
  const ScalarInts table = (ScalarInts)(a.table + (long long)it.seq * a.max_pages);
  const uint32_t sK_lds = (uint32_t)(uintptr_t)sK, sV_lds = (uint32_t)(uintptr_t)sV;
  const int key_last = it.held - 1;
  int k_off[CPT], v_off[CPT];
#pragma unroll
  for (int j = 0; j < CPT; ++j) {
    const int r = RPP * (wave + NW * j) + lane / UPR, u = lane % UPR;
    k_off[j] = (kWhole ? (lane / UPR) * ROWB : 0) + ((u ^ k_swizzle<D>(r)) * 16);
    v_off[j] = (kWhole ? (lane / UPR) * ROWB : 0) + ((u ^ v_swizzle<D>(r)) * 16);
  }
  // the pages of a tile's pieces, asked for one step before they are needed: of a piece's first key and, !kWhole, of its last
  struct Pages { int first[CPT], last[kWhole ? 1 : CPT]; };
  auto ask = [&](Pages& p, int start) {
#pragma unroll
    for (int j = 0; j < CPT; ++j) {
      const int key = start + RPP * (wave + NW * j);
      p.first[j] = table[div_page(a, __builtin_amdgcn_readfirstlane(min(key, key_last)))];
      if constexpr (!kWhole) p.last[j] = table[div_page(a, __builtin_amdgcn_readfirstlane(min(key, key_last - (RPP - 1)) + (RPP - 1)))];
    }
  };
  // the tile that starts at key `start` into the LDS at `slot`; keys that are none read as zeros
  auto request = [&](uint64_t pool, const Pages& p, uint32_t slot, int start, const int (&off)[CPT]) {
#pragma unroll
    for (int j = 0; j < CPT; ++j) {
      const uint32_t dst = __builtin_amdgcn_readfirstlane(slot + (wave + NW * j) * 1024);
      const int key = __builtin_amdgcn_readfirstlane(start + RPP * (wave + NW * j)), left = min(RPP, it.held - key);
      const int entry = div_page(a, min(key, key_last)), inside = key - entry * a.page;
      if constexpr (kWhole) {
        const int id = p.first[j];
        const bool ok = left > 0 && is_page(a, id);
        const uint64_t base = ok ? pool + (uint64_t)(uint32_t)id * page_bytes + (uint32_t)inside * ROWB : pool;
        const i32x4 desc = {__builtin_amdgcn_readfirstlane((int)(uint32_t)base), __builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32)),
                            __builtin_amdgcn_readfirstlane(ok ? left * ROWB : 0), 0x00020000};
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :: "s"(dst), "v"(off[j]), "s"(desc) : "memory", "m0");
      } else {
        // two pages at most, or (pages shorter than a piece) a look at the table by every lane
        const int i = lane / UPR;
        int id = p.first[j], at = inside + i;
        if (a.page >= RPP - 1) {
          if (at >= a.page) { at -= a.page; id = p.last[j]; }
        } else {
          const int e = div_page(a, min(key + i, max(key_last, 0)));
          id = a.table[(long long)it.seq * a.max_pages + e];
          at = key + i - e * a.page;
        }
        const uint64_t from = i < left && is_page(a, id) ? pool + (uint64_t)(uint32_t)id * page_bytes + (uint32_t)(at * ROWB + off[j])
                                                         : reinterpret_cast<uint64_t>(zero_row);
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(dst), "v"(from) : "memory", "m0");
      }
    }
  };

  // ---- LDS reads.  K fragment of step s: unit 2 s + h of row l32.  V^T fragment (feature 32 dt + l32; keys 16 t2 + 8 y + 4 h .. + 3) by
  // transposing reads: a 16-lane group fetches 4 keys x 16 features in chunks of 8 bytes
  uint32_t k_addr[NS], v_addr[ND][2];
#pragma unroll
  for (int s = 0; s < NS; ++s) k_addr[s] = l32 * ROWB + 16 * ((2 * s + h) ^ k_swizzle<D>(l32));
  {
    const int j16 = lane & 15, g16 = (lane >> 4) & 1, key = 4 * h + (j16 >> 2);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int y = 0; y < 2; ++y)   // (the swizzles of rows 16 apart agree)
        v_addr[dt][y] = (key + 8 * y) * ROWB + 16 * ((4 * dt + 2 * g16 + ((j16 & 3) >> 1)) ^ v_swizzle<D>(key + 8 * y)) + 8 * (j16 & 1);
  }

  f32x16 o[ND];
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.0f;
  float m_ref = -INFINITY, l_run = 0.0f;
  uint32_t seen = 0;
  bool odd = false;   // values that are not finite lie next to rows that do not see them: they were left out (uniform)

  // uniform: does any row of the wavefront see a key of the tile, does every row see all of them
  auto some_of = [&](int start) { return active && start < view_hi.hi && (start + kKeyTile > view_lo.lo || start < view.sink); };
  auto all_of = [&](int start) {
    return start + kKeyTile <= view_lo.hi && (start >= view_hi.lo || start + kKeyTile <= view.sink) && !bad_pages;
  };
  // the tile's keys that lie in pages, a bit each
  auto existing = [&](int start) {
    if (!bad_pages) return 0xffffffffu;
    const int key = start + l32;
    return (uint32_t)__ballot(key < it.held && is_page(a, a.table[(long long)it.seq * a.max_pages + div_page(a, min(key, key_last))]));
  };

  int start0 = start_of(0), start1 = start_of(1), start2 = start_of(2), start3 = start_of(3);   // of tiles i .. i + 3
  Pages kp, vp;                                                                                // of tiles i + 3 and i + 1
  // the rows have to be here before the first request: the compiler does not count requests, and a wait behind them would be one for
  // all of them
#pragma unroll
  for (int s = 0; s < NS; ++s) asm volatile("" : "+v"(qf[s]));
  if (count > 0) {
    Pages p0, p2;
    ask(p0, start0);
    ask(vp, start1);
    ask(p2, start2);
    ask(kp, start3);
    request(k_pool, p0, sK_lds, start0, k_off);
    request(v_pool, p0, sV_lds, start0, v_off);
    request(k_pool, vp, sK_lds + TILE, start1, k_off);
    request(k_pool, p2, sK_lds + 2 * TILE, start2, k_off);
  }
  asm volatile("s_waitcnt vmcnt(%0)" :: "n"(3 * CPT) : "memory");
  if (NW > 1) __syncthreads();
  bf16x8 kf[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) kf[s] = *reinterpret_cast<const bf16x8*>(sK + k_addr[s]);

  // tile i: its K fragments are in registers; slot_next, slot_new: where K of tiles i + 1 and i + 3 lie; par: V slot of tile i
  auto step = [&](int i, const int slot_next, const int slot_new, const int par) {
    const int start = start0;
    const bool some = some_of(start);
    f32x16 sacc;
    if (some) {
#pragma unroll
      for (int r = 0; r < 16; ++r) sacc[r] = 0.0f;
#pragma unroll
      for (int s = 0; s < NS; ++s) sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s], qf[s], sacc, 0, 0, 0);
    }
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(CPT) : "memory");   // K of tile i + 1 and V of tile i; K of i + 2 may fly
    if (NW > 1) __syncthreads();
    request(v_pool, vp, sV_lds + (par ^ 1) * TILE, start1, v_off);
    auto v_frag = [&](int dt, int t2) {
      const char* p = sV + v_addr[dt][0] + par * TILE + 16 * ROWB * t2;
      const char* q = sV + v_addr[dt][1] + par * TILE + 16 * ROWB * t2;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(p));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(q));
      const s16x8 both = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      return __builtin_bit_cast(bf16x8, both);
    };
    bf16x8 vf[ND], vg[ND], pf[2];
    if (some) {
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) vf[dt] = v_frag(dt, 0);
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) vg[dt] = v_frag(dt, 1);
    }
#pragma unroll
    for (int s = 0; s < NS; ++s) kf[s] = *reinterpret_cast<const bf16x8*>(sK + k_addr[s] + slot_next * TILE);
    __builtin_amdgcn_sched_barrier(0);
    if (some) {
      if (!all_of(start)) {
        const uint32_t sees = view.sees_tile(start) & existing(start), mine = sees >> (4 * h);
        seen |= sees;
#pragma unroll
        for (int r = 0; r < 16; ++r) sacc[r] = masked_score(sacc[r], mine, 8 * (r >> 2) + (r & 3));
        // a probability of zero does not make a NaN or an infinity vanish: such values become zero here
        uint32_t cut = 0;
        auto finite = [&](bf16x8& v) {
          u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const u16x2 left = __builtin_bit_cast(u16x2, 0x7f807f80u - (w[e] & 0x7f807f80u)), one = {1, 1}, zero = {0, 0};
            const uint32_t keep = __builtin_bit_cast(uint32_t, (u16x2)(zero - __builtin_elementwise_min(left, one)));   // all ones where finite
            cut |= ~keep;
            w[e] &= keep;
          }
          v = __builtin_bit_cast(bf16x8, w);
        };
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) { finite(vf[dt]); finite(vg[dt]); }
        odd = odd || __any(cut != 0);
      } else {
        seen = 1;
      }
      // ---- online softmax in the exp2 domain
      float mx = max3f(max3f(max3f(sacc[0], sacc[1], sacc[2]), max3f(sacc[3], sacc[4], sacc[5]), max3f(sacc[6], sacc[7], sacc[8])),
                       max3f(sacc[9], sacc[10], sacc[11]), max3f(sacc[12], sacc[13], max3f(sacc[14], sacc[15], sacc[15])));
      {
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        mx = max3f(__uint_as_float(sw[0]), __uint_as_float(sw[1]), __uint_as_float(sw[1])) * a.c_scale;
      }
      // every row by its own maximum: what the other rows of the wavefront see is nothing to it
      const bool grows = mx > m_ref + kGrow;
      if (__any(grows)) {
        const float m_new = grows ? mx : m_ref;
        const float alpha = grows ? __builtin_amdgcn_exp2f(m_ref - m_new) : 1.0f;
        m_ref = m_new;
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
      }
      const float m_use = m_ref == -INFINITY ? 0.0f : m_ref;
      float psum = 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = __builtin_amdgcn_exp2f(fmaf(sacc[r], a.c_scale, -m_use));
        psum += p;
        pf[r >> 3][r & 7] = static_cast<__bf16>(p);
      }
      l_run += psum;
      // ---- O^T += V^T P^T
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[dt], pf[0], o[dt], 0, 0, 0);
    }
    request(k_pool, kp, sK_lds + slot_new * TILE, start3, k_off);   // (between the products: requests in a row queue up)
    if (some) {
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vg[dt], pf[1], o[dt], 0, 0, 0);
    }
    start0 = start1;
    start1 = start2;
    start2 = start3;
    start3 = start_of(i + 4);
    ask(vp, start1);
    ask(kp, start3);
  };
  if constexpr (KSLOTS == 4) {
    for (int i = 0; i < count; i += 4) {
      step(i, 1, 3, 0);
      if (i + 1 >= count) break;
      step(i + 1, 2, 0, 1);
      if (i + 2 >= count) break;
      step(i + 2, 3, 1, 0);
      if (i + 3 >= count) break;
      step(i + 3, 0, 2, 1);
    }
  } else {
    int slot = 0;
    for (int i = 0; i < count; ++i) {   // (the step that frees slot i mod 3 fills it with tile i + 3)
      const int next = slot == 2 ? 0 : slot + 1;
      step(i, next, slot, i & 1);
      slot = next;
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing may land on the sums
  if (NW > 1) __syncthreads();

  // ---- the values that were left out, in the rows that see them: infinite, or NaN next to a probability of zero.  Off the fast path:
  // key by key, straight from the pages
  if (odd) {
    const float m_use = m_ref == -INFINITY ? 0.0f : m_ref;
#pragma unroll 1
    for (int i = 0; i < count; ++i) {
      const int start = start_of(i);
      if (!some_of(start) || all_of(start)) continue;
#pragma unroll 1
      for (int k = 0; k < kKeyTile; ++k) {
        const int key = start + k;
        if (key >= it.held) break;
        const int entry = div_page(a, key), id = table[entry];
        if (!is_page(a, id)) continue;
        const uint64_t at = (uint64_t)(uint32_t)id * page_bytes + (uint32_t)(key - entry * a.page) * ROWB;
        float s = 0.0f;
#pragma unroll
        for (int c = 0; c < NS; ++c) {
          const bf16x8 w = *reinterpret_cast<const bf16x8*>(k_pool + at + 2 * (16 * c + 8 * h));
#pragma unroll
          for (int e = 0; e < 8; ++e) s = fmaf(static_cast<float>(w[e]), static_cast<float>(qf[c][e]), s);
        }
        s += __shfl_xor(s, 32, kWave);
        const bool sees = view.sees(key), positive = __builtin_amdgcn_exp2f(fmaf(s, a.c_scale, -m_use)) > 0.0f;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const uint2 w = *reinterpret_cast<const uint2*>(v_pool + at + 2 * (32 * dt + 8 * q + 4 * h));
            const uint32_t v[4] = {w.x << 16, w.x & 0xffff0000u, w.y << 16, w.y & 0xffff0000u};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (sees && (v[e] & 0x7f800000u) == 0x7f800000u) o[dt][4 * q + e] += positive ? __uint_as_float(v[e]) : __builtin_nanf("");
          }
      }
    }
  }

  // ---- the sums of the wavefront's rows go to LDS
  {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
    l_run = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    if (seen != 0 && m_ref == -INFINITY && l_run == 0.0f) l_run = kOnlyInfinite;
    float* const row = reinterpret_cast<float*>(sK) + (32 * wave + l32) * (D + 4);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(row + 32 * dt + 8 * q + 4 * h) = make_float4(o[dt][4 * q], o[dt][4 * q + 1], o[dt][4 * q + 2], o[dt][4 * q + 3]);
    if (h == 0) *reinterpret_cast<float2*>(reinterpret_cast<float*>(sK) + BM * (D + 4) + 2 * (32 * wave + l32)) = make_float2(m_ref, l_run);
  }
  finish_item<bf16_t, D, BM, KS, S::NT>(
      a, sc, it, [&](int u) { return reinterpret_cast<const float*>(smem + u * S::SPAN); },
      [&](int u) { return reinterpret_cast<const float*>(smem + u * S::SPAN) + BM * (D + 4); }, reinterpret_cast<int*>(smem + S::FLAG));
}

// ---- launches
struct Plan { int rows, items, target, cmin, capacity; };   // rows of a workgroup

constexpr int kComputeUnits = 256;

Plan plan_of(const hf_paged& c, int n_q) {
  const int group = c.heads / c.heads_kv;
  Plan p;
  // a workgroup of 128 rows where a sequence has more than 32 on the average
  p.rows = (long long)n_q * group > 32ll * c.n_seqs ? 128 : 32;
  const long long tiles = ((long long)n_q * group / p.rows + (n_q < c.n_seqs ? n_q : c.n_seqs)) * c.heads_kv;   // (at most)
  p.target = (p.rows == 128 ? 4 : 2) * kComputeUnits;
  p.cmin = p.rows == 128 ? 16 : 8;
  const long long key_tiles = ((long long)c.max_pages * c.page_tokens + kKeyTile - 1) / kKeyTile;
  const long long most = (key_tiles + p.cmin - 1) / p.cmin;             // parts of a row tile
  long long items = tiles + p.target, parts = 2 * p.target + 64;
  if (items > tiles * most) items = tiles * most;
  if (parts > tiles * most) parts = tiles * most;
  p.items = (int)((items + 7) & ~7ll);
  p.capacity = most > 1 ? (int)parts : 0;
  return p;
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

template <int D, int NW, int KS, bool kWhole> int launch(const PagedAttnArgs& a, const PagedSchedule& sc, int items, hipStream_t s) {
  using S = Shape<D, NW, KS>;
  static LdsGrant grant;
  const int rc = grant_lds(grant, reinterpret_cast<const void*>(&paged_attn_kernel<D, NW, KS, kWhole>), S::LDS, "hf_paged_attn_fwd");
  if (rc != HF_OK) return rc;
  hipLaunchKernelGGL((paged_attn_kernel<D, NW, KS, kWhole>), dim3(items), dim3(S::NT), S::LDS, s, a, sc);
  return check_launch("hf_paged_attn_fwd");
}

template <int D> int launch_of(const PagedAttnArgs& a, const PagedSchedule& sc, const Plan& p, hipStream_t s) {
  const bool whole = a.page % (512 / D) == 0;
  if (p.rows == 128) return whole ? launch<D, 4, 1, true>(a, sc, p.items, s) : launch<D, 4, 1, false>(a, sc, p.items, s);
  return whole ? launch<D, 1, 4, true>(a, sc, p.items, s) : launch<D, 1, 4, false>(a, sc, p.items, s);
}

}  // namespace

size_t paged_workspace_bytes(const hf_paged& c, int n_q) {
  if (n_q == 0) return 0;
  const Plan p = plan_of(c, n_q);
  if (p.capacity == 0) return 0;
  return align256((size_t)p.capacity * 8) + align256((size_t)p.capacity * p.rows * (c.head_dim + 2) * 4);
}

int launch_paged_attn(const hf_paged& c, PagedAttnArgs a, void* workspace, hipStream_t s) {
  const Plan p = plan_of(c, a.n_q);
  int shift = 0;
  while ((1 << shift) < c.page_tokens) ++shift;
  a.page_shift = 31 + shift;
  a.page_magic = (uint32_t)((1ull << a.page_shift) / (unsigned)c.page_tokens + 1);
  PagedSchedule sc = {};
  sc.target = p.target;
  sc.cmin = p.cmin;
  sc.capacity = p.capacity;
  sc.by_xcd = p.rows == 128;
  if (p.capacity > 0) {
    sc.counters = static_cast<unsigned long long*>(workspace);
    sc.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + align256((size_t)p.capacity * 8));
    sc.tag = next_call_tag();
  }
  if (c.dtype == HF_F32) return launch_paged_attn_f32(c, a, sc, p.rows, p.items, s);
  return c.head_dim == 128 ? launch_of<128>(a, sc, p, s) : launch_of<64>(a, sc, p, s);
}

}  // namespace hf
