// Attention over a cache of pages in fp32 (hf_paged_attn_fwd, fp32 storage): both products on v_mfma_f32_32x32x2_f32.
//
// Rows, items and statistics as in hf_paged_attn.hip (the instruction's result has the same layout).  A lane's operands are 16-byte pieces of
// its key's row (product over features), and of every value row the 16 or 8 bytes that hold its features (product over keys).  The four k
// indices of a piece feed four instructions; accumulator e holds the features E * (row of the result) + e.  Every key has an address of its
// own, so that pages may end anywhere; a key that is none reads a row of zeros.
//   NW 4, KS 1   128 rows, tiles of 32 keys go global -> LDS directly, a tile ahead, one barrier each; two workgroups or more a compute unit
//                share its matrix cores.  16 heads x 4096 x 4096, head_dim 128: 124 TFLOP/s of the 154 that a matrix product reaches, the
//                matrix cores 78 % of the cycles busy; the rest is vector work, which fp32 products leave little room beside them.
//                (With tiles that every wavefront reads for itself a prompt of 2048 tokens, 8 heads, took 152 us, now 120)
//   NW 1, KS 4   32 rows, bound by memory: every wavefront reads its own tiles from memory to registers.  32 sequences of 4096 tokens,
//                8 heads: 220 us, 4.9 TB/s
//   NW 1, KS 1   the same, a row tile a wavefront, for many sequences (300 of 25 to 500 tokens: 178 us, by four wavefronts each 258)
#include "hf_paged_attn.h"

namespace hf {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
#define HF_GLOBAL __attribute__((address_space(1)))   // (of an address that went from lane to lane the compiler would not know)

namespace {

__device__ float zero_row_f32[128];

__device__ __forceinline__ bool not_finite(float v) { return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u; }

template <int D, int NW, int KS>
__global__ __launch_bounds__(64 * NW * KS, NW > 1 ? 2 : 1) void paged_attn_f32_kernel(const PagedLaunch) {
  static_assert(NW == 1 || KS == 1, "groups share no barrier");
  constexpr int BM = 32 * NW, NT = 64 * NW * KS, NC = D / 8, E = D / 32;   // a lane's pieces of a key; features of its piece of a value
  constexpr int ROWB = 4 * D, TILE = kKeyTile * ROWB, RPP = 1024 / ROWB, UPR = ROWB / 16;   // (LDS: keys of a 1 KB request, 16-byte units of a key)
  constexpr int SPAN = BM * (D + 4) + BM * 2;                              // a group's sums and statistics, in floats
  extern __shared__ __attribute__((aligned(16))) float sums[];
  typedef float piece __attribute__((ext_vector_type(E)));

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
  const int wave = wave_in_wg % NW, grp = wave_in_wg / NW;
  const int l32 = lane & 31, h = lane >> 5, group = a.group;

  const int x_last = it.first + it.rows - 1, x = min(it.first + 32 * wave + l32, x_last), token = div_group(a, x);
  const RowView view = row_view(a, it, token);
  const bool active = 32 * wave < it.rows;
  const RowView view_lo = row_view(a, it, div_group(a, min(it.first + 32 * wave, x_last)));
  const RowView view_hi = row_view(a, it, div_group(a, min(it.first + 32 * wave + 31, x_last)));
  f32x4 qf[NC];
  {
    const float* q = static_cast<const float*>(a.Q) + (long long)(it.begin + token) * a.qt +
                     (long long)(it.head_kv * group + (x - token * group)) * a.qh + 4 * h;
#pragma unroll
    for (int c = 0; c < NC; ++c) qf[c] = *reinterpret_cast<const f32x4*>(q + 8 * c);
  }
  f32x16 o[E];
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[e][r] = 0.0f;
  float m_ref = -INFINITY, l_run = 0.0f;
  uint32_t seen = 0;

  const bool bad_pages = any_bad_page(a, it);
  const int count = active || NW > 1 ? max(0, (it.t1 - it.t0 - grp + KS - 1) / KS) : 0;
  auto start_of = [&](int i) { return kKeyTile * it.keys.tile(it.t0 + grp + KS * i); };   // (page_tiles = 0)
  auto some_of = [&](int start) { return start < view_hi.hi && (start + kKeyTile > view_lo.lo || start < view.sink); };
  auto all_of = [&](int start) {
    return start + kKeyTile <= view_lo.hi && (start >= view_hi.lo || start + kKeyTile <= view.sink) && !bad_pages;
  };
  // the lane's key of a tile: its page (-1: none, or past the cache)
  const int32_t* const table = a.table + (long long)it.seq * a.max_pages;
  auto page_of = [&](int i) {
    const int key = i < count ? start_of(i) + l32 : it.held;
    const int id = table[div_page(a, min(key, max(it.held - 1, 0)))];
    return key < it.held && is_page(a, id) ? id : -1;
  };
  const long long page_rows = (long long)a.heads_kv * a.page, head_row = (long long)it.head_kv * a.page;
  auto offset_of = [&](int i, int id) {   // element offset in the pool
    const int key = start_of(i) + l32;
    return (id * page_rows + head_row + (key - div_page(a, key) * a.page)) * D;
  };
  // ---- NW 1: registers
  auto load_keys = [&](f32x4 (&k)[NC], int i, int id) {
    const uintptr_t p = reinterpret_cast<uintptr_t>((id >= 0 ? static_cast<const float*>(a.K_pages) + offset_of(i, id) : zero_row_f32) + 4 * h);
#pragma unroll
    for (int c = 0; c < NC; ++c) k[c] = *(const HF_GLOBAL f32x4*)(p + 32 * c);
  };
  // ---- NW 4: two slots of a K and a V tile; unit u of key row r sits at u ^ r (modulo the row) in K, so that 8 lanes read 8 places
  typedef __attribute__((address_space(3))) char* Lds;
  const uint32_t lds = (uint32_t)(uintptr_t)(Lds)(char*)sums;
  auto request = [&](int i, int id) {
    const long long at = id >= 0 ? offset_of(i, id) * 4 : -1;
    const uint32_t slot = lds + (i & 1) * 2 * TILE;
#pragma unroll
    for (int j = 0; j < kKeyTile / RPP / NW; ++j) {
      const int piece_at = wave + NW * j, r = RPP * piece_at + lane / UPR, u = lane % UPR;
      const long long row = __shfl(at, r, kWave);
      const uint64_t zeros = reinterpret_cast<uint64_t>(zero_row_f32);
      const uint64_t k = row >= 0 ? reinterpret_cast<uint64_t>(a.K_pages) + row + 16 * (u ^ (r % UPR)) : zeros;
      const uint64_t v = row >= 0 ? reinterpret_cast<uint64_t>(a.V_pages) + row + 16 * u : zeros;
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                   :: "s"(__builtin_amdgcn_readfirstlane(slot + 1024 * piece_at)), "v"(k) : "memory", "m0");
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                   :: "s"(__builtin_amdgcn_readfirstlane(slot + TILE + 1024 * piece_at)), "v"(v) : "memory", "m0");
    }
  };
  if constexpr (NW > 1) {   // the rows have to be here before the first request, which the compiler does not count: a wait behind it would be
#pragma unroll              // one for it as well
    for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(qf[c]));
  }
  int id = -1, id_next = -1;
  f32x4 kf[NC];
  if (count > 0) {
    id = page_of(0);
    id_next = page_of(1);
    if constexpr (NW > 1) request(0, id);
    else load_keys(kf, 0, id);
  }
  bool odd = false;   // values that are not finite lie next to rows that do not see them: they were left out (uniform)

#pragma unroll 1
  for (int i = 0; i < count; ++i) {
    const int start = start_of(i);
    const uint32_t exists = (uint32_t)__ballot(id >= 0);
    const int id_after = page_of(i + 2);
    if constexpr (NW > 1) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // tile i, requested a tile ago
      __syncthreads();                                    // of everybody, and the other slot is free
      if (i + 1 < count) request(i + 1, id_next);
    }
    if (active && some_of(start)) {
      piece vf[16];   // (NW 4: read four at a time, next to the products of the four before)
      auto read_values = [&](int r) {
        const float* const v_row = sums + (i & 1) * (TILE / 2) + TILE / 4 + 4 * h * D + E * l32;
#pragma unroll
        for (int n = 0; n < 4; ++n) vf[r + n] = *reinterpret_cast<const piece*>(v_row + (2 * r + n) * D);
      };
      // a probability of zero does not make a NaN or an infinity vanish: where rows are masked, such values become zero
      auto cut_values = [&](int r0, int n) {
        auto full = [](float v) { return ((__float_as_uint(v) & 0x7f800000u) + 0x00800000u) & 0x80000000u; };   // the top bit: its exponent is full
        uint32_t any = 0;
#pragma unroll
        for (int r = r0; r < r0 + n; ++r)
#pragma unroll
          for (int e = 0; e < E; ++e) any |= full(vf[r][e]);
        if (!__any(any != 0)) return;
        odd = true;
#pragma unroll
        for (int r = r0; r < r0 + n; ++r)
#pragma unroll
          for (int e = 0; e < E; ++e) vf[r][e] = __uint_as_float(__float_as_uint(vf[r][e]) & ~(uint32_t)((int)full(vf[r][e]) >> 31));
      };
      const bool masked = !all_of(start);
      f32x16 sacc;
#pragma unroll
      for (int r = 0; r < 16; ++r) sacc[r] = 0.0f;
      if constexpr (NW > 1) {
        const float* const k_row = sums + (i & 1) * (TILE / 2) + l32 * D;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const f32x4 k = *reinterpret_cast<const f32x4*>(k_row + 4 * ((2 * c + h) ^ (l32 % UPR)));
#pragma unroll
          for (int e = 0; e < 4; ++e) sacc = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], qf[c][e], sacc, 0, 0, 0);
        }
        read_values(0);
      } else {
        const float* const v_row = id >= 0 ? static_cast<const float*>(a.V_pages) + offset_of(i, id) : zero_row_f32;
        auto row_of = [&](int key) { return (uintptr_t)__shfl((unsigned long long)reinterpret_cast<uintptr_t>(v_row), key, kWave); };   // of the tile
#pragma unroll
        for (int r = 0; r < 16; ++r) vf[r] = *(const HF_GLOBAL piece*)(row_of(8 * (r >> 2) + 4 * h + (r & 3)) + 4 * E * l32);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) sacc = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[c][e], qf[c][e], sacc, 0, 0, 0);
        if (i + 1 < count) load_keys(kf, i + 1, id_next);
      }
      if (masked) {
        const uint32_t sees = view.sees_tile(start) & exists, mine = sees >> (4 * h);
        seen |= sees;
#pragma unroll
        for (int r = 0; r < 16; ++r) sacc[r] = masked_score(sacc[r], mine, 8 * (r >> 2) + (r & 3));
        if constexpr (NW == 1) cut_values(0, 16);
      } else {
        seen = 1;
      }
      float mx = sacc[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sacc[r]);
      mx = fmaxf(mx, __shfl_xor(mx, 32, kWave)) * a.c_scale;
      const bool grows = mx > m_ref;
      if (__any(grows)) {
        const float m_new = grows ? mx : m_ref;
        const float alpha = grows ? __builtin_amdgcn_exp2f(m_ref - m_new) : 1.0f;
        m_ref = m_new;
        l_run *= alpha;
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[e][r] *= alpha;
      }
      const float m_use = m_ref == -INFINITY ? 0.0f : m_ref;
      float psum = 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        sacc[r] = __builtin_amdgcn_exp2f(fmaf(sacc[r], a.c_scale, -m_use));
        psum += sacc[r];
      }
      l_run += psum;
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        if constexpr (NW > 1) {
          if (masked) cut_values(r, 4);
          if (r < 12) read_values(r + 4);
        }
#pragma unroll
        for (int n = r; n < r + 4; ++n)
#pragma unroll
          for (int e = 0; e < E; ++e) o[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[n][e], sacc[n], o[e], 0, 0, 0);
      }
    } else if (NW == 1 && i + 1 < count) {
      load_keys(kf, i + 1, id_next);
    }
    id = id_next;
    id_next = id_after;
  }

  // ---- the values that were left out, in the rows that see them: infinite, or NaN next to a probability of zero
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
        const long long at = (id * page_rows + head_row + (key - entry * a.page)) * D;
        const float *kr = static_cast<const float*>(a.K_pages) + at, *vr = static_cast<const float*>(a.V_pages) + at;
        float s = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const f32x4 w = *reinterpret_cast<const f32x4*>(kr + 8 * c + 4 * h);
#pragma unroll
          for (int e = 0; e < 4; ++e) s = fmaf(w[e], qf[c][e], s);
        }
        s += __shfl_xor(s, 32, kWave);
        const bool sees = view.sees(key), positive = __builtin_amdgcn_exp2f(fmaf(s, a.c_scale, -m_use)) > 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const piece w = *reinterpret_cast<const piece*>(vr + E * (8 * (r >> 2) + 4 * h + (r & 3)));
#pragma unroll
          for (int e = 0; e < E; ++e)
            o[e][r] += sees && not_finite(w[e]) ? (positive ? w[e] : __builtin_nanf("")) : 0.0f;
        }
      }
    }
  }

  if (NW > 1) __syncthreads();   // the tiles are done with; the sums take their place
  l_run += __shfl_xor(l_run, 32, kWave);
  if (seen != 0 && m_ref == -INFINITY && l_run == 0.0f) l_run = kOnlyInfinite;
  float* const row = sums + grp * SPAN + (32 * wave + l32) * (D + 4);
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    piece y;
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = o[e][r];
    *reinterpret_cast<piece*>(row + E * (8 * (r >> 2) + 4 * h + (r & 3))) = y;
  }
  if (h == 0) *reinterpret_cast<float2*>(sums + grp * SPAN + BM * (D + 4) + 2 * (32 * wave + l32)) = make_float2(m_ref, l_run);
  const PagedLaunch p = launch_arguments();
  finish_item<float, D, BM, KS, NT>(p.a, p.sc, it, [&](int u) { return sums + u * SPAN; }, [&](int u) { return sums + u * SPAN + BM * (D + 4); },
                                    reinterpret_cast<int*>(sums + KS * SPAN));
  if constexpr (NW > 1) return;
  }
}

template <int D, int NW, int KS> int launch(const PagedAttnArgs& a, const PagedSchedule& sc, int grid, hipStream_t s) {
  constexpr int kLds = KS * (32 * NW * (D + 4) + 64 * NW) * 4 + 16;
  static_assert(NW == 1 || 4 * kKeyTile * 4 * D <= kLds, "two slots of two tiles");
  static LdsGrant grant;
  const int rc = grant_lds(grant, reinterpret_cast<const void*>(&paged_attn_f32_kernel<D, NW, KS>), kLds, "hf_paged_attn_fwd");
  if (rc != HF_OK) return rc;
  hipLaunchKernelGGL((paged_attn_f32_kernel<D, NW, KS>), dim3(grid), dim3(64 * NW * KS), kLds, s, PagedLaunch{a, sc});
  return check_launch("hf_paged_attn_fwd");
}

}  // namespace

int launch_paged_attn_f32(const hf_paged& c, const PagedAttnArgs& a, const PagedSchedule& sc, int rows, int ks, int grid, hipStream_t s) {
  if (rows == 128) return c.head_dim == 128 ? launch<128, 4, 1>(a, sc, grid, s) : launch<64, 4, 1>(a, sc, grid, s);
  if (ks == 1) return c.head_dim == 128 ? launch<128, 1, 1>(a, sc, grid, s) : launch<64, 1, 1>(a, sc, grid, s);
  return c.head_dim == 128 ? launch<128, 1, 4>(a, sc, grid, s) : launch<64, 1, 4>(a, sc, grid, s);
}

}  // namespace hf
