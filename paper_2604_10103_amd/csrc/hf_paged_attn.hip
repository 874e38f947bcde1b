// Attention over a cache of pages on bf16 MFMA (hf_paged_attn_fwd, bf16 storage, head_dim 64 or 128).
//
// The layout of the window kernels (hf_attn_mfma.hip): a wavefront owns 32 rows, tiles of 32 keys, both products transposed,
//   S^T (keys x rows) = K_tile (A, from LDS) x Q^T (B, registers),   O^T (d x rows) += V_tile^T (A, LDS) x P^T (B, registers),
// so that the statistics of a row are private to its two lanes and the exponentials of S^T are, rounded to bf16, the B operand of the
// second product.  K and V tiles go global -> LDS directly, V^T fragments are transposing reads, three K slots and two V slots.
// Here the rows are tokens x heads of a group, and a tile lies in pages: its descriptor is scalar arithmetic on an entry of the page table
// that the scalar unit fetched a step before.
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
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

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

// kBig: pages of 32 tokens and more: a tile lies in one page (one descriptor) or in two (an address per lane).  Else every piece of a tile
// has a page of its own, or, where that ends inside a piece, every lane.
template <int D, int NW, int KS, bool kBig>
__global__ __launch_bounds__(64 * NW * KS, (NW == 4 ? 2 : 1)) void paged_attn_kernel(const PagedLaunch) {
  static_assert(NW == 1 || KS == 1, "groups share no barrier");
  using S = Shape<D, NW, KS>;
  constexpr int BM = S::BM, ROWB = S::ROWB, TILE = S::TILE, KSLOTS = S::KSLOTS;
  constexpr int RPP = 1024 / ROWB, UPR = ROWB / 16;       // keys of a 1 KB piece, 16-byte units of a key
  constexpr int CPT = kKeyTile / RPP / NW;                // pieces of a tile that a wavefront requests
  constexpr int NS = D / 16, ND = D / 32;                 // steps of S^T, 32-feature blocks of O^T
  extern __shared__ __attribute__((aligned(16))) char smem[];

  PagedItem it;
  {
    const PagedLaunch p = launch_arguments();
    if (!find_item<BM>(p.a, p.sc, blockIdx.x, it)) return;
  }
  const PagedAttnArgs a = launch_arguments().a;

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
  auto start_of = [&](int i) { return i < count ? it.keys.start(it.t0 + grp + KS * i) : kNone; };

  // ---- requests: 1 KB pieces; piece j of this wavefront is the tile's keys RPP (wave + NW j) ..
  const uint32_t page_rows = (uint32_t)a.heads_kv * (uint32_t)a.page, head_rows = (uint32_t)it.head_kv * (uint32_t)a.page;   // (of the pool: < 2^32)
  const uint64_t k_pool = reinterpret_cast<uint64_t>(a.K_pages), v_pool = reinterpret_cast<uint64_t>(a.V_pages);
  const ScalarInts table = (ScalarInts)(a.table + (long long)it.seq * a.max_pages);
  const uint32_t sK_lds = (uint32_t)(uintptr_t)sK, sV_lds = (uint32_t)(uintptr_t)sV;
  const int key_last = it.held - 1;
  auto row_at = [&](int id, int inside) { return (uint64_t)((uint32_t)id * page_rows + head_rows + (uint32_t)inside) * ROWB; };
  int k_off[CPT], v_off[CPT];
#pragma unroll
  for (int j = 0; j < CPT; ++j) {
    const int r = RPP * (wave + NW * j) + lane / UPR, u = lane % UPR;
    const int row = kBig ? r * ROWB : 0;   // (from the tile's first key, or none: a lane's place in its piece is added where it is needed)
    k_off[j] = row + ((u ^ k_swizzle<D>(r)) * 16);
    v_off[j] = row + ((u ^ v_swizzle<D>(r)) * 16);
  }
  auto to_lds_from = [&](uint32_t dst, uint64_t from) {   // every lane from an address of its own
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :: "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(from) : "memory", "m0");
  };
  auto to_lds = [&](uint32_t dst, int off, uint64_t base, int bytes) {   // from a buffer, behind whose end there are zeros
    const i32x4 desc = {__builtin_amdgcn_readfirstlane((int)(uint32_t)base), __builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32)),
                        __builtin_amdgcn_readfirstlane(bytes), 0x00020000};
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" :: "s"(dst), "v"(off), "s"(desc) : "memory", "m0");
  };
  const uint64_t zeros = reinterpret_cast<uint64_t>(zero_row);

  // The pages of a tile are asked for one step before its K is requested, its V is requested two steps after that.
  // kBig: what was asked for (page, place in it) and what came of it (byte offset in the pool; bytes, -1: two pages)
  struct Asked { int id[kBig ? 1 : CPT], inside; };
  struct Place { uint64_t at; int bytes; };
  auto ask = [&](Asked& p, int start) {
    if constexpr (kBig) {
      const int key = min(start, key_last), entry = div_page(a, key);
      p.id[0] = table[entry];
      p.inside = key - entry * a.page;
    } else {
#pragma unroll
      for (int j = 0; j < CPT; ++j) p.id[j] = table[div_page(a, min(start + RPP * (wave + NW * j), key_last))];
    }
  };
  auto place_of = [&](const Asked& p, int start) {
    const int left = min(max(it.held - start, 0), kKeyTile);
    Place q;
    q.at = is_page(a, p.id[0]) ? row_at(p.id[0], p.inside) : 0;
    q.bytes = p.inside + left > a.page ? -1 : (is_page(a, p.id[0]) ? left * ROWB : 0);
    return q;
  };
  // the tile that starts at key `start` into the LDS at `slot`; keys that are none read as zeros
  auto request_big = [&](uint64_t pool, const Place& q, uint32_t slot, int start, const int (&off)[CPT]) {
    if (q.bytes >= 0) {   // (uniform)
#pragma unroll
      for (int j = 0; j < CPT; ++j) to_lds(slot + (wave + NW * j) * 1024, off[j], pool + q.at, q.bytes);
    } else {
      const int entry = div_page(a, start), cut = (entry + 1) * a.page - start;
      const int id0 = table[entry], id1 = table[entry + 1];   // (there are keys behind the cut)
      const uint64_t base0 = is_page(a, id0) ? pool + row_at(id0, start - entry * a.page) : zeros;
      const uint64_t base1 = is_page(a, id1) ? pool + row_at(id1, 0) - (uint64_t)(uint32_t)(cut * ROWB) : zeros;
#pragma unroll
      for (int j = 0; j < CPT; ++j) {
        const int r = RPP * (wave + NW * j) + lane / UPR;
        const bool ok = start + r < it.held && is_page(a, r < cut ? id0 : id1);
        to_lds_from(slot + (wave + NW * j) * 1024, ok ? (r < cut ? base0 : base1) + (uint32_t)off[j] : zeros);
      }
    }
  };
  auto request_small = [&](uint64_t pool, const Asked& p, uint32_t slot, int start, const int (&off)[CPT]) {
    const int i = lane / UPR;
#pragma unroll
    for (int j = 0; j < CPT; ++j) {
      const uint32_t dst = slot + (wave + NW * j) * 1024;
      const int key = start + RPP * (wave + NW * j), left = min(RPP, it.held - key);
      if (a.page % RPP == 0) {   // (uniform) the piece lies in one page
        const int entry = div_page(a, min(key, key_last)), id = p.id[j];
        const bool ok = left > 0 && is_page(a, id);
        to_lds(dst, i * ROWB + off[j], ok ? pool + row_at(id, key - entry * a.page) : pool, ok ? left * ROWB : 0);
      } else {
        const int mine = min(key + i, max(key_last, 0)), entry = div_page(a, mine), id = a.table[(long long)it.seq * a.max_pages + entry];
        to_lds_from(dst, i < left && is_page(a, id) ? pool + row_at(id, mine - entry * a.page) + (uint32_t)off[j] : zeros);
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

  // Tiles by what the wavefront's rows see of them, in ranges of i (uniform): of those behind the sink's, every row sees all keys of
  // i_all .. i_all + n_all - 1; none sees any of those before i_some and behind i_end
  const int i_window = max(0, (it.keys.s1 - it.t0 - grp + KS - 1) / KS);   // the first tile behind the sink's
  auto first_from = [&](int key) {   // the first i >= i_window whose tile starts at `key` or behind
    const int t = (key + kKeyTile - 1) / kKeyTile - it.keys.skip;
    return max(i_window, (t - it.t0 - grp + KS - 1 + KS * 0x100000) / KS - 0x100000);
  };
  const int i_some = first_from(view_lo.lo - (kKeyTile - 1)), i_end = active ? min(count, first_from(view_hi.hi)) : 0;
  const int i_all = first_from(view_hi.lo), n_all = bad_pages ? 0 : max(0, first_from(view_lo.hi - (kKeyTile - 1)) - i_all);
  auto some_of = [&](int i) { return i < i_end && (i >= i_some || i < i_window); };
  auto all_of = [&](int i) { return (unsigned)(i - i_all) < (unsigned)n_all; };
  // the tile's keys that lie in pages, a bit each
  auto existing = [&](int start) {
    if (!bad_pages) return 0xffffffffu;
    const int key = start + l32;
    return (uint32_t)__ballot(key < it.held && is_page(a, a.table[(long long)it.seq * a.max_pages + div_page(a, min(key, key_last))]));
  };

  // the rows have to be here before the first request: the compiler does not count requests, and a wait behind them would be one for
  // all of them
#pragma unroll
  for (int s = 0; s < NS; ++s) asm volatile("" : "+v"(qf[s]));
  int start1 = start_of(1), start2 = start_of(2), start3 = start_of(3);   // of tiles i + 1 .. i + 3
  Asked asked_v, asked_k;                                                 // !kBig: tiles i + 1 and i + 3; kBig: asked_k is tile i + 4's
  Place place1, place2, place3;                                           // kBig: of tiles i + 1 .. i + 3
  if (count > 0) {
    const int start0 = start_of(0);
    if constexpr (kBig) {
      Asked p0, p1, p2, p3;
      ask(p0, start0);
      ask(p1, start1);
      ask(p2, start2);
      ask(p3, start3);
      ask(asked_k, start_of(4));
      const Place place0 = place_of(p0, start0);
      place1 = place_of(p1, start1);
      place2 = place_of(p2, start2);
      place3 = place_of(p3, start3);
      request_big(k_pool, place0, sK_lds, start0, k_off);
      request_big(v_pool, place0, sV_lds, start0, v_off);
      request_big(k_pool, place1, sK_lds + TILE, start1, k_off);
      request_big(k_pool, place2, sK_lds + 2 * TILE, start2, k_off);
    } else {
      Asked p0, p2;
      ask(p0, start0);
      ask(asked_v, start1);
      ask(p2, start2);
      ask(asked_k, start3);
      request_small(k_pool, p0, sK_lds, start0, k_off);
      request_small(v_pool, p0, sV_lds, start0, v_off);
      request_small(k_pool, asked_v, sK_lds + TILE, start1, k_off);
      request_small(k_pool, p2, sK_lds + 2 * TILE, start2, k_off);
    }
  }
  asm volatile("s_waitcnt vmcnt(%0)" :: "n"(3 * CPT) : "memory");
  if (NW > 1) __syncthreads();
  bf16x8 kf[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) kf[s] = *reinterpret_cast<const bf16x8*>(sK + k_addr[s]);

  // tile i: its K fragments are in registers; slot_next, slot_new: where K of tiles i + 1 and i + 3 lie; par: V slot of tile i
  auto step = [&](int i, const int slot_next, const int slot_new, const int par) {
    const bool some = some_of(i);
    f32x16 sacc;
    if (some) {
#pragma unroll
      for (int r = 0; r < 16; ++r) sacc[r] = 0.0f;
#pragma unroll
      for (int s = 0; s < NS; ++s) sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s], qf[s], sacc, 0, 0, 0);
    }
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(CPT) : "memory");   // K of tile i + 1 and V of tile i; K of i + 2 may fly
    if (NW > 1) __syncthreads();
    if constexpr (kBig) request_big(v_pool, place1, sV_lds + (par ^ 1) * TILE, start1, v_off);
    else request_small(v_pool, asked_v, sV_lds + (par ^ 1) * TILE, start1, v_off);
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
      if (!all_of(i)) {
        const int start = start_of(i);
        const uint32_t sees = view.sees_tile(start) & existing(start), mine = sees >> (4 * h);
        seen |= sees;
#pragma unroll
        for (int r = 0; r < 16; ++r) sacc[r] = masked_score(sacc[r], mine, 8 * (r >> 2) + (r & 3));
        // a probability of zero does not make a NaN or an infinity vanish: such values become zero here
        auto full = [](uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; };   // a half's top bit: its exponent is full
        uint32_t any = 0;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
          for (int e = 0; e < 4; ++e) any |= full(__builtin_bit_cast(u32x4, vf[dt])[e]) | full(__builtin_bit_cast(u32x4, vg[dt])[e]);
        if (__any(any != 0)) {
          odd = true;
          auto clear = [&](bf16x8& v) {
            u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t c = full(w[e]);
              w[e] &= ~(c | (c - (c >> 15)));
            }
            v = __builtin_bit_cast(bf16x8, w);
          };
#pragma unroll
          for (int dt = 0; dt < ND; ++dt) { clear(vf[dt]); clear(vg[dt]); }
        }
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
    // (between the products: requests in a row queue up)
    if constexpr (kBig) request_big(k_pool, place3, sK_lds + slot_new * TILE, start3, k_off);
    else request_small(k_pool, asked_k, sK_lds + slot_new * TILE, start3, k_off);
    if (some) {
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vg[dt], pf[1], o[dt], 0, 0, 0);
    }
    start1 = start2;
    start2 = start3;
    start3 = start_of(i + 4);
    if constexpr (kBig) {
      place1 = place2;
      place2 = place3;
      place3 = place_of(asked_k, start3);
      ask(asked_k, start_of(i + 5));
    } else {
      ask(asked_v, start1);
      ask(asked_k, start3);
    }
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
      if (!some_of(i) || all_of(i)) continue;
      const int start = start_of(i);
#pragma unroll 1
      for (int k = 0; k < kKeyTile; ++k) {
        const int key = start + k;
        if (key >= it.held) break;
        const int entry = div_page(a, key), id = table[entry];
        if (!is_page(a, id)) continue;
        const uint64_t at = row_at(id, key - entry * a.page);
        float s = 0.0f;
#pragma unroll
        for (int c = 0; c < NS; ++c) {
          const bf16x8 w = *(const __attribute__((address_space(1))) bf16x8*)(k_pool + at + 2 * (16 * c + 8 * h));
#pragma unroll
          for (int e = 0; e < 8; ++e) s = fmaf(static_cast<float>(w[e]), static_cast<float>(qf[c][e]), s);
        }
        s += __shfl_xor(s, 32, kWave);
        const bool sees = view.sees(key), positive = __builtin_amdgcn_exp2f(fmaf(s, a.c_scale, -m_use)) > 0.0f;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const u32x2 w = *(const __attribute__((address_space(1))) u32x2*)(v_pool + at + 2 * (32 * dt + 8 * q + 4 * h));
            const uint32_t v[4] = {w[0] << 16, w[0] & 0xffff0000u, w[1] << 16, w[1] & 0xffff0000u};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              o[dt][4 * q + e] += sees && (v[e] & 0x7f800000u) == 0x7f800000u ? (positive ? __uint_as_float(v[e]) : __builtin_nanf("")) : 0.0f;
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
  const PagedLaunch p = launch_arguments();
  finish_item<bf16_t, D, BM, KS, S::NT>(
      p.a, p.sc, it, [&](int u) { return reinterpret_cast<const float*>(smem + u * S::SPAN); },
      [&](int u) { return reinterpret_cast<const float*>(smem + u * S::SPAN) + BM * (D + 4); }, reinterpret_cast<int*>(smem + S::FLAG));
}

// ---- launches
struct Plan {
  int rows, items, capacity;   // rows of a workgroup
  PagedSchedule sc;
};

Plan plan_of(const hf_paged& c, int n_q) {
  const int group = c.heads / c.heads_kv;
  Plan p = {};
  // a workgroup of 128 rows where a sequence has more than 32 on the average
  p.rows = (long long)n_q * group > 32ll * c.n_seqs ? 128 : 32;
  if (p.rows == 128) {
    p.sc.target = 1536;
    p.sc.tile = p.sc.tile_alone = 0.535f;
    p.sc.start = 3.0f;
    p.sc.meet = 6.0f;
    p.sc.join = 0.5f;
  } else {
    p.sc.target = 1024;
    p.sc.tile = 0.8f;
    p.sc.tile_alone = 0.22f;
    p.sc.start = 4.0f;
    p.sc.meet = 5.0f;
    p.sc.join = 0.1f;
  }
  p.sc.by_xcd = p.rows == 128;
  const long long tiles = ((long long)n_q * group / p.rows + (n_q < c.n_seqs ? n_q : c.n_seqs)) * c.heads_kv;   // (at most)
  const long long key_tiles = ((long long)c.max_pages * c.page_tokens + kKeyTile - 1) / kKeyTile;
  const long long most = key_tiles < 1024 ? key_tiles : 1024;           // parts of a row tile
  long long items = tiles + p.sc.target, parts = 2 * p.sc.target + 64;
  if (items > tiles * most) items = tiles * most;
  if (parts > tiles * most) parts = tiles * most;
  p.items = (int)((items + 7) & ~7ll);
  p.capacity = most > 1 ? (int)parts : 0;
  return p;
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

template <int D, int NW, int KS, bool kBig> int launch(const PagedAttnArgs& a, const PagedSchedule& sc, int items, hipStream_t s) {
  using S = Shape<D, NW, KS>;
  static LdsGrant grant;
  const int rc = grant_lds(grant, reinterpret_cast<const void*>(&paged_attn_kernel<D, NW, KS, kBig>), S::LDS, "hf_paged_attn_fwd");
  if (rc != HF_OK) return rc;
  hipLaunchKernelGGL((paged_attn_kernel<D, NW, KS, kBig>), dim3(items), dim3(S::NT), S::LDS, s, PagedLaunch{a, sc});
  return check_launch("hf_paged_attn_fwd");
}

template <int D> int launch_of(const PagedAttnArgs& a, const PagedSchedule& sc, const Plan& p, hipStream_t s) {
  const bool big = a.page >= kKeyTile;
  if (p.rows == 128) return big ? launch<D, 4, 1, true>(a, sc, p.items, s) : launch<D, 4, 1, false>(a, sc, p.items, s);
  return big ? launch<D, 1, 4, true>(a, sc, p.items, s) : launch<D, 1, 4, false>(a, sc, p.items, s);
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
  PagedSchedule sc = p.sc;
  sc.capacity = p.capacity;
  if (p.capacity > 0) {
    sc.counters = static_cast<unsigned long long*>(workspace);
    sc.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + align256((size_t)p.capacity * 8));
    sc.tag = next_call_tag();
  }
  if (c.dtype == HF_F32) return launch_paged_attn_f32(c, a, sc, p.rows, p.items, s);
  return c.head_dim == 128 ? launch_of<128>(a, sc, p, s) : launch_of<64>(a, sc, p, s);
}

}  // namespace hf
