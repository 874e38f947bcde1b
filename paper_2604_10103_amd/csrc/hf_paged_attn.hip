// Attention over a cache of pages on bf16 MFMA (hf_paged_attn_fwd, bf16 storage, head_dim 64 or 128).
//
// The layout of the window kernels (hf_attn_mfma.hip): a wavefront owns 32 rows, tiles of 32 keys, both products transposed,
//   S^T (keys x rows) = K_tile (A, from LDS) x Q^T (B, registers),   O^T (d x rows) += V_tile^T (A, LDS) x P^T (B, registers),
// so that the statistics of a row are private to its two lanes and the exponentials of S^T are, rounded to bf16, the B operand of the
// second product (that rounding, half a step of each probability, averages out over the keys: outputs are 0.0023 off 64 bits where exact
// probabilities leave 0.0017, the output's own rounding; a product of the remainders would double the second half of the matrix work).
// K and V tiles go global -> LDS directly, V^T fragments are transposing reads, three K slots (four where wavefronts share tiles) and two V
// slots.
// Here the rows are tokens x heads of a group, and a tile lies in a page.  A wavefront finds out for 64 tiles at once where they lie, a lane
// each; a tile's descriptor is then a few scalar instructions.  (12 heads x 4680 x 9360, pages of 1560: 287 us, with an address for every
// lane instead, as for pages of 16, 334; prompts of 2048 tokens over 6100 314 and 429.  Entries of the table that the scalar unit reads a tile ahead cost a sixth: they are on their way when the tile's
// barrier waits for everything that is; tiles that go on in the next page, and a branch for them, a tenth.)
//
// Four shapes of workgroup (NW wavefronts of rows, KS groups of wavefronts that share the keys):
//   NW 8, KS 1   256 rows, tiles shared by eight wavefronts, one barrier a tile, one workgroup a compute unit (head_dim 128): long chunks
//   NW 4, KS 1   128 rows, two workgroups a compute unit (head_dim 64: three): chunks
//   NW 1, KS 4   32 rows, every wavefront its own tiles and no barrier until the end: single tokens
//   NW 1, KS 1   the same by one wavefront, four workgroups a compute unit: single tokens of many sequences
// The first two are bound by matrix cores and softmax together, whose instructions a SIMD's two wavefronts issue one after the other, and by
// power: 12 heads x 4680 x 9360 reach 940 TFLOP/s at the 1.9 to 2.0 GHz that the chip holds there, the matrix cores 44 % of the cycles busy,
// the vector units 43 %, no LDS conflict.  (Wavefronts that take turns between barriers, one half at the products while the other is at its
// exponentials, need a third longer: alone, a wavefront leaves a fifth of the vector unit's issue slots empty.)  The others are bound by
// memory: 64 single tokens over 500 to 8191 keys in 211 us, 5.6 TB/s; short ones by the chain arguments, lengths, page table, keys
// (118 keys: 8.4 us, of which 3.3 go until the work is known, 1.5 until the rows are there, 1.4 for a tile, 1.0 for the end).
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

template <int D, int NW, int KS> struct Shape {
  static constexpr int BM = 32 * NW, NT = 64 * NW * KS;
  static constexpr int ROWB = 2 * D, TILE = kKeyTile * ROWB;
  static constexpr int KSLOTS = NW > 1 ? 4 : 3;
  static constexpr int GROUP = (KSLOTS + 2) * TILE;                  // a group's tiles: those of K, two of V
  static constexpr int OUT = BM * (D + 4) * 4 + BM * 8;              // a group's sums behind the loop, and its rows' statistics
  static constexpr int SPAN = GROUP > OUT ? GROUP : OUT;
  static constexpr int FLAG = GROUP > OUT ? OUT : KS * SPAN;         // an int behind the sums
  static constexpr int LDS = KS * SPAN + (GROUP > OUT ? 0 : 16);
};

// kBig: tiles end with their page: one descriptor a tile.  Else, where a page's last tile would be short too often, every lane has an address
// and pages may end anywhere.
template <int D, int NW, int KS, bool kBig>
__global__ __launch_bounds__(64 * NW * KS, (NW > 1 ? 2 : 1)) void paged_attn_kernel(const PagedLaunch) {
  static_assert(NW == 1 || KS == 1, "groups share no barrier");
  using S = Shape<D, NW, KS>;
  constexpr int BM = S::BM, ROWB = S::ROWB, TILE = S::TILE, KSLOTS = S::KSLOTS;
  constexpr int RPP = 1024 / ROWB, UPR = ROWB / 16;       // keys of a 1 KB piece, 16-byte units of a key
  constexpr int CPT = kKeyTile / RPP / NW;                // pieces of a tile that a wavefront requests
  constexpr int NS = D / 16, ND = D / 32;                 // steps of S^T, 32-feature blocks of O^T
  extern __shared__ __attribute__((aligned(16))) char smem[];

  PagedCursor cursor;
  {
    const PagedLaunch p = launch_arguments();
    cursor = first_item<BM, NW == 1>(p.a, p.sc);
  }
  for (bool again = false;; again = true) {
  PagedItem it;
  {
    const PagedLaunch p = launch_arguments();
    if (!next_item<BM, NW == 1>(p.a, p.sc, cursor, it)) return;
  }
  if (again) __syncthreads();   // everybody is done with the sums in LDS
  const PagedAttnArgs a = launch_arguments().a;

  const int tid = thread_id(), lane = tid & 63;
  const int wave_in_wg = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave = KS == 1 ? wave_in_wg : 0, grp = KS == 1 ? 0 : wave_in_wg;
  char* const sK = smem + grp * S::SPAN;
  const int l32 = lane & 31, h = lane >> 5, group = a.group;

  // ---- this lane's row (past the item's rows: its last one again; only the rows that there are get stored)
  const int x_last = it.first + it.rows - 1, x = min(it.first + 32 * wave + l32, x_last), token = div_group(a, x);
  const RowView view = row_view(a, it, token);
  const bool active = 32 * wave < it.rows;                 // (uniform)
  // what all rows of the wavefront see, and what any of them sees
  const RowView view_lo = row_view(a, it, div_group(a, min(it.first + 32 * wave, x_last)));
  const RowView view_hi = row_view(a, it, div_group(a, min(it.first + 32 * wave + 31, x_last)));
  bf16x8 qf[NS];
  {
    const bf16_t* q = static_cast<const bf16_t*>(a.Q) + (long long)(it.begin + token) * a.qt +
                      (long long)(it.head_kv * group + (x - token * group)) * a.qh + 8 * h;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(q + 16 * s);
  }
  const bool bad_pages = kBig ? false : any_bad_page(a, it);   // (kBig: such a tile has no bytes)

  // ---- the group's tiles, every wavefront of it the same: every KS-th of the item's, or (pages by lane) a run of them, whose pages are fewer
  constexpr int kStride = kBig ? KS : 1;
  const int run = (it.t1 - it.t0 + KS - 1) / KS, base_tile = it.t0 + grp * (kBig ? 1 : run);
  const int count = kBig ? max(0, (it.t1 - base_tile + KS - 1) / KS) : max(0, min(run, it.t1 - base_tile));
  auto start_of = [&](int i) { return tile_start(a, it.keys.tile(base_tile + kStride * i)); };   // (0 <= i < count)

  // ---- requests: 1 KB pieces; piece j of this wavefront is the tile's keys RPP (wave + NW j) ..  Keys that are none read as zeros
  const uint32_t page_rows = (uint32_t)a.heads_kv * (uint32_t)a.page, head_rows = (uint32_t)it.head_kv * (uint32_t)a.page;   // (of the pool: < 2^32)
  const uint64_t k_pool = reinterpret_cast<uint64_t>(a.K_pages), v_pool = reinterpret_cast<uint64_t>(a.V_pages);
  const int32_t* const table = a.table + (long long)it.seq * a.max_pages;
  typedef __attribute__((address_space(3))) char* Lds;
  const uint32_t sK_lds = (uint32_t)(uintptr_t)(Lds)smem + grp * S::SPAN, sV_lds = sK_lds + KSLOTS * TILE;
  const int key_last = it.held - 1;
  const uint64_t zeros = reinterpret_cast<uint64_t>(zero_row);
  int k_off[CPT], v_off[CPT];
#pragma unroll
  for (int j = 0; j < CPT; ++j) {
    const int r = RPP * (wave + NW * j) + lane / UPR, u = lane % UPR;
    const int row = kBig ? r * ROWB : 0;   // (from the tile's first key; by lane: the key's own row is added)
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
  auto pool_row = [&](int id, int inside) { return (uint32_t)id * page_rows + head_rows + (uint32_t)inside; };

  // kBig: where 64 tiles lie, a lane each: the pool's row of the first key, and how many bytes.  Of the tiles that K is requested for, and of
  // those that V is, which come two later
  struct Places { uint32_t row; int bytes; };
  Places k_places = {0, 0}, v_places = {0, 0};
  auto find_places = [&](int i0) {
    const int i = i0 + lane, start = i < count ? start_of(i) : it.held;
    k_places = {0, 0};
    if (start < it.held) {
      const int entry = div_page(a, start), inside = start - entry * a.page, id = table[entry];
      k_places.row = pool_row(id, inside);
      k_places.bytes = is_page(a, id) ? min(min(it.held - start, a.page - inside), kKeyTile) * ROWB : 0;
    }
  };
  auto request_big = [&](uint64_t pool, const Places& p, int i, uint32_t slot, const int (&off)[CPT]) {   // its bytes
    const int bytes = __builtin_amdgcn_readlane(p.bytes, i & 63);
    const uint64_t base = pool + (uint64_t)(uint32_t)__builtin_amdgcn_readlane(p.row, i & 63) * ROWB;
#pragma unroll
    for (int j = 0; j < CPT; ++j) to_lds(slot + (wave + NW * j) * 1024, off[j], base, bytes);
    return bytes;
  };
  // else: the pool's row of the lane's key (the tile's key lane % 32), kNoRow: none; of tiles i + 1 .. i + 3.  The wavefront keeps 64 entries
  // of the table, from ids_base on, a lane each
  constexpr uint32_t kNoRow = 0xffffffffu;
  uint32_t row1 = kNoRow, row2 = kNoRow, row3 = kNoRow;
  int ids = -1, ids_base = -kWave;
  const int entry_last = it.held > 0 ? div_page(a, key_last) : 0;
  auto rows_of = [&](int i) {
    const int start = i < count ? start_of(i) : it.held;
    if (start >= it.held) return kNoRow;   // (uniform)
    const int first = div_page(a, start), last = div_page(a, min(start + kKeyTile - 1, key_last));
    if (first < ids_base || last >= ids_base + kWave) {
      ids_base = first;
      ids = first + lane <= entry_last ? table[first + lane] : -1;
    }
    const int key = min(start + l32, key_last), entry = div_page(a, key), id = __shfl(ids, entry - ids_base, kWave);
    return start + l32 < it.held && is_page(a, id) ? pool_row(id, key - entry * a.page) : kNoRow;
  };
  auto request_rows = [&](uint64_t pool, uint32_t rows, uint32_t slot, const int (&off)[CPT]) {
#pragma unroll
    for (int j = 0; j < CPT; ++j) {
      const uint32_t row = (uint32_t)__shfl((int)rows, RPP * (wave + NW * j) + lane / UPR, kWave);
      to_lds_from(slot + (wave + NW * j) * 1024, row != kNoRow ? pool + (uint64_t)row * ROWB + (uint32_t)off[j] : zeros);
    }
  };
  // V of tile i + 1 and K of tile i + 3, whose turn it is in step i
  int bytes_next = 0;   // kBig: of the tile whose V was requested last
  auto request_v = [&](int i, uint32_t slot) {
    if constexpr (kBig) {
      if (((i + 1) & 63) == 0) v_places = k_places;
      bytes_next = request_big(v_pool, v_places, i + 1, slot, v_off);
    } else {
      request_rows(v_pool, row1, slot, v_off);
    }
  };
  auto request_k = [&](int i, uint32_t slot) {
    if constexpr (kBig) {
      if (((i + 3) & 63) == 0) find_places(i + 3);
      request_big(k_pool, k_places, i + 3, slot, k_off);
    } else {
      request_rows(k_pool, row3, slot, k_off);
      row1 = row2;
      row2 = row3;
      row3 = rows_of(i + 4);
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
        v_addr[dt][y] = sV_lds + (key + 8 * y) * ROWB + 16 * ((4 * dt + 2 * g16 + ((j16 & 3) >> 1)) ^ v_swizzle<D>(key + 8 * y)) + 8 * (j16 & 1);
  }

  f32x16 o[ND];
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.0f;
  float m_ref = -INFINITY, l_run = 0.0f;
  uint32_t seen = 0;
  bool odd = false;   // values that are not finite lie next to rows that do not see them: they were left out (uniform)

  // the tiles of which every row of the wavefront sees all keys (uniform): i_all .. i_all + n_all - 1, behind the sink's
  auto index_of = [&](int tile) {   // the first i at that tile (of those behind the sink's) or behind it
    const int t = max(it.keys.s1, tile - it.keys.skip) - base_tile;
    return t <= 0 ? 0 : (t + kStride - 1) / kStride;
  };
  const int i_all = index_of(tiles_to(a, view_hi.lo)), n_all = bad_pages ? 0 : max(0, index_of(tile_of(a, view_lo.hi)) - i_all);
  auto all_of = [&](int i) { return (unsigned)(i - i_all) < (unsigned)n_all; };
  // the tile's keys that are there, a bit each
  auto existing = [&](int start, int bytes) {
    if constexpr (kBig) return RowView::below(bytes / ROWB);
    if (!bad_pages) return 0xffffffffu;
    const int key = start + l32;
    return (uint32_t)__ballot(key < it.held && is_page(a, table[div_page(a, min(key, key_last))]));
  };

  // the rows have to be here before the first request: the compiler does not count requests, and a wait behind them would be one for
  // all of them
  if constexpr (kBig) find_places(0);
#pragma unroll
  for (int s = 0; s < NS; ++s) asm volatile("" : "+v"(qf[s]));
  if (count > 0) {
    if constexpr (kBig) {
      v_places = k_places;
      request_big(k_pool, k_places, 0, sK_lds, k_off);
      bytes_next = request_big(v_pool, k_places, 0, sV_lds, v_off);
      request_big(k_pool, k_places, 1, sK_lds + TILE, k_off);
      request_big(k_pool, k_places, 2, sK_lds + 2 * TILE, k_off);
    } else {
      const uint32_t row0 = rows_of(0);
      row1 = rows_of(1);
      row2 = rows_of(2);
      row3 = rows_of(3);
      request_rows(k_pool, row0, sK_lds, k_off);
      request_rows(v_pool, row0, sV_lds, v_off);
      request_rows(k_pool, row1, sK_lds + TILE, k_off);
      request_rows(k_pool, row2, sK_lds + 2 * TILE, k_off);
    }
  }
  asm volatile("s_waitcnt vmcnt(%0)" :: "n"(3 * CPT) : "memory");
  if (NW > 1) __syncthreads();
  bf16x8 kf[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) kf[s] = *reinterpret_cast<const bf16x8*>(sK + k_addr[s]);

  // tile i: its K fragments are in registers; slot_next, slot_new: where K of tiles i + 1 and i + 3 lie; par: V slot of tile i
  auto step = [&](int i, const int slot_next, const int slot_new, const int par) {
    const int bytes = bytes_next;
    f32x16 sacc;
#pragma unroll
    for (int r = 0; r < 16; ++r) sacc[r] = 0.0f;
#pragma unroll
    for (int s = 0; s < NS; ++s) sacc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s], qf[s], sacc, 0, 0, 0);
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(CPT) : "memory");   // K of tile i + 1 and V of tile i; K of i + 2 may fly
    if (NW > 1) __syncthreads();
    request_v(i, sV_lds + (par ^ 1) * TILE);
    auto v_frag = [&](int dt, int t2) {
      const uint32_t at = par * TILE + 16 * ROWB * t2;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(uintptr_t)(v_addr[dt][0] + at));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(uintptr_t)(v_addr[dt][1] + at));
      const s16x8 both = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      return __builtin_bit_cast(bf16x8, both);
    };
    bf16x8 vf[ND], vg[ND], pf[2];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) vf[dt] = v_frag(dt, 0);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) vg[dt] = v_frag(dt, 1);
#pragma unroll
    for (int s = 0; s < NS; ++s) kf[s] = *reinterpret_cast<const bf16x8*>(sK + k_addr[s] + slot_next * TILE);
    __builtin_amdgcn_sched_barrier(0);
    {
      if (!all_of(i) || (kBig && bytes < TILE)) {
        const int start = start_of(i);
        const uint32_t sees = view.sees_tile(start) & existing(start, bytes), mine = sees >> (4 * h);
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
      // (a row with a NaN keeps its reference: its sum is NaN in any case)
      float mx = max_of3(max_of3(max_of3(sacc[0], sacc[1], sacc[2]), max_of3(sacc[3], sacc[4], sacc[5]), max_of3(sacc[6], sacc[7], sacc[8])),
                         max_of3(sacc[9], sacc[10], sacc[11]), max_of3(sacc[12], sacc[13], max_of3(sacc[14], sacc[15], sacc[15])));
      {
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        mx = max_of3(__uint_as_float(sw[0]), __uint_as_float(sw[1]), __uint_as_float(sw[1])) * a.c_scale;
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
    request_k(i, sK_lds + slot_new * TILE);   // (between the products: requests in a row queue up)
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vg[dt], pf[1], o[dt], 0, 0, 0);
  };
  if constexpr (NW == 1) {
    int slot = 0;
    for (int i = 0; i < count; ++i) {   // (the step that frees slot i mod 3 fills it with tile i + 3)
      const int next = slot == 2 ? 0 : slot + 1;
      step(i, next, slot, i & 1);
      slot = next;
    }
  } else if (active) {
    for (int i = 0; i < count; i += 4) {
      step(i, 1, 3, 0);
      if (i + 1 >= count) break;
      step(i + 1, 2, 0, 1);
      if (i + 2 >= count) break;
      step(i + 2, 3, 1, 0);
      if (i + 3 >= count) break;
      step(i + 3, 0, 2, 1);
    }
  } else {   // no rows: the wavefront only carries its share of the tiles
    for (int i = 0; i < count; ++i) {
      asm volatile("s_waitcnt vmcnt(%0)" :: "n"(CPT) : "memory");
      __syncthreads();
      request_v(i, sV_lds + ((i & 1) ^ 1) * TILE);
      request_k(i, sK_lds + ((i + 3) & 3) * TILE);
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
      const int start = start_of(i), tile_end = kBig ? min(start + kKeyTile, (div_page(a, start) + 1) * a.page) : start + kKeyTile;
      if (all_of(i) && tile_end == start + kKeyTile) continue;
#pragma unroll 1
      for (int key = start; key < min(tile_end, it.held); ++key) {
        const int entry = div_page(a, key), id = table[entry];
        if (!is_page(a, id)) continue;
        const uint64_t at = (uint64_t)pool_row(id, key - entry * a.page) * ROWB;
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
  if constexpr (NW > 1) return;
  }
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
  // A workgroup of 128 rows where a sequence has more than 32 on the average.  256 rows, whose tiles travel half as often, take 0.89 us a
  // tile where two workgroups of 128 take 1.07, if a compute unit's rounds of them are no more (12 heads x 4680 x 9360: 287 and 293 us;
  // over a window of 9360 and a sink frame 415 and 430; a prompt of 4096, 32 heads on 8: 157 and 158).  The times are fits to launches of 128 to 768 row tiles over 256 to 4096 keys.
  p.rows = rows > 32ll * c.n_seqs ? 128 : 32;
  if (p.rows == 128 && c.dtype == HF_BF16 && c.head_dim == 128 && rows > 128ll * c.n_seqs) {
    const long long n = (rows + c.n_seqs - 1) / c.n_seqs, heads = (long long)c.n_seqs * c.heads_kv;   // (as if all were as long)
    auto rounds = [&](int of) { return (double)(((n + of - 1) / of * heads + 255) / 256); };
    if (rounds(256) * 0.89 <= rounds(128) * 0.535) p.rows = 256;
  }
  p.ks = p.rows == 32 ? 4 : 1;
  p.sc.units = 256.0f;
  // A row tile a wavefront where there are enough for all: its chain (rows, page table, first keys) then passes next to three others'.  512
  // sequences of 13 to 250 keys, 8 key heads: 100 us, with four wavefronts a row tile 192; 256 of 150 to 3000: 308 and 305; 128 of 400 to
  // 8000: 397 and 378
  if (p.rows == 32 && tiles(32) >= 1024) {
    p.ks = 1;
    p.sc.groups = 1024;
    p.sc.units = 1024.0f;
    const float bytes = (c.head_dim == 128 ? 1.0f : 0.5f) * (c.dtype == HF_F32 ? 2.0f : 1.0f);
    p.sc.tile = 2.8f * bytes;
    p.sc.tile_alone = 1.9f * bytes;
    p.sc.start = 4.0f;
    p.sc.meet = 5.0f;
    p.sc.join = 0.1f;
    p.sc.lead = 2;
  } else if (p.rows == 32) {
    p.sc.groups = 256;
    p.sc.tile = 0.8f;
    p.sc.tile_alone = 0.27f;
    p.sc.start = 4.0f;
    p.sc.meet = 5.0f;
    p.sc.join = 0.1f;
    p.sc.lead = 5;
  } else {
    const bool wide = c.head_dim == 128;
    p.sc.groups = 65536 / p.rows;   // (at most 512)
    p.sc.meet = 6.0f;
    p.sc.join = 1.0f;
    p.sc.start = 5.0f;
    if (c.dtype == HF_F32) {
      p.sc.tile = wide ? 4.35f : 2.35f;
      p.sc.tile_alone = wide ? 4.66f : 2.9f;
      p.sc.start = 9.0f;
    } else if (p.rows == 256) {
      p.sc.tile = p.sc.tile_alone = 0.89f;
      p.sc.start = 9.0f;
    } else {
      p.sc.tile = wide ? 0.535f : 0.29f;
      p.sc.tile_alone = wide ? 0.7f : 0.4f;
    }
  }
  const long long key_tiles = (long long)c.max_pages * ((c.page_tokens + kKeyTile - 1) / kKeyTile);   // (at most)
  long long grid = p.rows == 32 ? p.sc.groups : tiles(p.rows) + p.sc.groups;
  if (grid > tiles(p.rows) * key_tiles) grid = tiles(p.rows) * key_tiles;
  p.grid = (int)((grid + 7) & ~7ll);
  p.sc.meets = key_tiles > 1;
  return p;
}

// n / d = n * magic >> shift (the result) for n < 2^31
int magic_of(int d, uint32_t& magic) {
  int bits = 0;
  while ((1 << bits) < d) ++bits;
  magic = (uint32_t)((1ull << (31 + bits)) / (unsigned)d + 1);
  return 31 + bits;
}

// The counters' part of every workspace is as large, whatever the call: what a call of another shape left there are counters of its tag
constexpr size_t kCounterBytes = 2 * 1024 * 8;

template <int D, int NW, int KS, bool kBig> int launch(const PagedAttnArgs& a, const PagedSchedule& sc, int grid, hipStream_t s) {
  using S = Shape<D, NW, KS>;
  static LdsGrant grant;
  const int rc = grant_lds(grant, reinterpret_cast<const void*>(&paged_attn_kernel<D, NW, KS, kBig>), S::LDS, "hf_paged_attn_fwd");
  if (rc != HF_OK) return rc;
  hipLaunchKernelGGL((paged_attn_kernel<D, NW, KS, kBig>), dim3(grid), dim3(S::NT), S::LDS, s, PagedLaunch{a, sc});
  return check_launch("hf_paged_attn_fwd");
}

template <int D> int launch_of(const PagedAttnArgs& a, const PagedSchedule& sc, const Plan& p, hipStream_t s) {
  const bool big = a.page_tiles > 0;
  if constexpr (D == 128) {
    if (p.rows == 256) return big ? launch<D, 8, 1, true>(a, sc, p.grid, s) : launch<D, 8, 1, false>(a, sc, p.grid, s);
  }
  if (p.rows == 128) return big ? launch<D, 4, 1, true>(a, sc, p.grid, s) : launch<D, 4, 1, false>(a, sc, p.grid, s);
  if (p.ks == 1) return big ? launch<D, 1, 1, true>(a, sc, p.grid, s) : launch<D, 1, 1, false>(a, sc, p.grid, s);
  return big ? launch<D, 1, 4, true>(a, sc, p.grid, s) : launch<D, 1, 4, false>(a, sc, p.grid, s);
}

}  // namespace

long long paged_threads(const hf_paged& c, int n_q) {
  const Plan p = plan_of(c, n_q);
  return (long long)p.grid * (2 * p.rows * p.ks);   // 64 for 32 rows, times the groups
}

size_t paged_workspace_bytes(const hf_paged& c, int n_q) {
  if (n_q == 0) return 0;
  const Plan p = plan_of(c, n_q);
  if (!p.sc.meets) return 0;
  return kCounterBytes + (size_t)p.sc.groups * 2 * p.rows * (c.head_dim + 2) * 4;
}

int launch_paged_attn(const hf_paged& c, PagedAttnArgs a, void* workspace, hipStream_t s) {
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
  // tiles that end with their page where the last, short ones are a sixteenth at most (pages of 16 keys would halve every tile)
  const int tiles = (c.page_tokens + kKeyTile - 1) / kKeyTile;
  if (c.dtype == HF_BF16 && tiles * kKeyTile * 16 <= c.page_tokens * 17) {
    a.page_tiles = tiles;
    a.tiles_shift = magic_of(tiles, a.tiles_magic);
  }
  if (c.dtype == HF_F32) return launch_paged_attn_f32(c, a, sc, p.rows, p.ks, p.grid, s);
  return c.head_dim == 128 ? launch_of<128>(a, sc, p, s) : launch_of<64>(a, sc, p, s);
}

}  // namespace hf
