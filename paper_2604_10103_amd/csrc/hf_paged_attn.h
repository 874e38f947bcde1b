// Attention over a cache of pages: what its kernels share (internal).
//
// Rows.  The query heads of a group read the same keys, so a sequence's rows are numbered token by token, head by head of the group:
// row x of (sequence, key head h) is token x / group, query head h * group + x % group.  A workgroup takes BM of them.
//
// Work.  The grid is fixed by what the host knows; what a workgroup does follows from the lengths, which only the device knows: every
// wavefront derives it for itself from cu_new and seq_lens, 64 sequences at a time, without exchange.  Keys count in tiles of 32.
//
//   pieces  A row tile that sees w tiles is cut into ceil(w / C) parts of equal length, C = ceil(longest w / S); a workgroup takes a (key
//           head, sequence, part, rows).  S is the best of 64 candidates, one a lane, by a model of the launch: with n = the
//           work in row tiles as long as the longest and x = n S / units,
//               rounds(x) (longest w / S * t(x) + start) + (S > 1 ? meet + join S : 0)  microseconds,
//           rounds(x) = x rounded up where all pieces are as long, else x + 1/2 (single tokens: 3/4), and t(x) what a tile takes: `tile`
//           where the units are full, and next to an idle half of them more (chunks) or, bound by memory, less (single tokens) than its
//           share.  Only S with n S <= groups are looked at, and S = 1.
//   shares  (few rows, where no two workgroups read the same keys) All row tiles of all key heads lie on one line, each as long as its
//           key tiles (between a sequence's first and last row tile they are taken to grow evenly) and `lead` more for what its start
//           costs; each of `groups` workgroups gets an equal share of the line.  A share's end that falls near a row tile's ends moves
//           there.  So a workgroup has whole row tiles and at most two parts.
// Where workgroups of 32 rows have work for more than one round, shares are taken if the model expects them to be faster: 64 single
// tokens over 500 to 8191 keys 211 us, in pieces 278.  Rows of chunks read the same keys at the same time when they lie in pieces, and
// find them in the L2; in shares they do not (4680 rows of 12 heads over 9360 keys take an eighth longer).  Nor does it pay to cut off
// what the longest rows have over the others: 4680 rows that see 10920 to 14040 keys take 6 to 11 % longer with 14 to 22 % of these cut off.
// A single token over 4096 keys takes 15 us in parts, 34 whole; four over 131071 keys 108 and 1130.
//
// Parts of a row meet in the workspace: each writes its sums (fp32) there, the last one to arrive adds them in the order of the parts.
#pragma once

#include <type_traits>

#include "hf_paged.h"

namespace hf {

constexpr int kKeyTile = 32;

struct PagedSchedule {
  int groups;                    // workgroups that may be parts of a row tile's work (32 rows: the grid, if there is work for so many)
  int lead;
  bool meets;                    // there is a workspace: 2 groups parts, and as many counters
  float tile, tile_alone;        // microseconds a tile takes where the chip is full, and alone on a compute unit
  float start, meet, join;
  float units;                   // workgroups that work at a time: the compute units, or four a unit
  unsigned long long* counters;  // [2 groups] arrivals at a row tile
  float* parts;                  // [2 groups][BM][D], behind them [2 groups][BM][2]: row maximum and sum
  unsigned long long tag;
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

// the thread's number, as if unknown before: what follows from it is formed anew in every phase instead of being kept over the others
__device__ __forceinline__ int thread_id() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// ---- pages, and tiles of keys.  A tile is 32 keys from a multiple of 32 on, or, page_tiles given, of a page: its last tile may be short
__device__ __forceinline__ bool is_page(const PagedAttnArgs& a, int id) { return (unsigned)id < (unsigned)a.n_pages; }
__device__ __forceinline__ int div_page(const PagedAttnArgs& a, int key) {   // key / a.page for 0 <= key < 2^31
  return (int)(((unsigned long long)(unsigned)key * a.page_magic) >> a.page_shift);
}
__device__ __forceinline__ int div_tiles(const PagedAttnArgs& a, int tile) {
  return (int)(((unsigned long long)(unsigned)tile * a.tiles_magic) >> a.tiles_shift);
}
__device__ __forceinline__ int div_group(const PagedAttnArgs& a, int row) {
  return (int)(((unsigned long long)(unsigned)row * a.group_magic) >> a.group_shift);
}
__device__ __forceinline__ int tile_of(const PagedAttnArgs& a, int key) {   // that holds the key
  if (a.page_tiles == 0) return key / kKeyTile;
  const int page = div_page(a, key);
  return page * a.page_tiles + (key - page * a.page) / kKeyTile;
}
__device__ __forceinline__ int tiles_to(const PagedAttnArgs& a, int key) { return key > 0 ? tile_of(a, key - 1) + 1 : 0; }   // that hold keys before it
__device__ __forceinline__ int tile_start(const PagedAttnArgs& a, int tile) {
  if (a.page_tiles == 0) return kKeyTile * tile;
  const int page = div_tiles(a, tile);
  return page * a.page + kKeyTile * (tile - page * a.page_tiles);
}

// the key tiles of some rows: 0 .. s1 - 1 (sink), then from s1 + skip on; n of them
struct KeyTiles {
  int s1, skip, n;
  __device__ __forceinline__ int tile(int t) const { return t < s1 ? t : t + skip; }
};

// tokens t_lo .. t_hi of a sequence with m new tokens and `len` in all, of which `held` can lie in the cache
__device__ __forceinline__ KeyTiles key_tiles(const PagedAttnArgs& a, int m, int len, int held, int t_lo, int t_hi) {
  const int p_lo = len - m + t_lo, p_hi = len - m + t_hi;
  const int end = a.causal ? max(0, min(held, p_hi + 1)) : held;
  const int w1 = tiles_to(a, end);
  KeyTiles k = {0, 0, w1};
  if (a.window > 0) {
    const long long first = (long long)p_lo - a.window + 1;
    const int w0 = first <= 0 ? 0 : (first >= end ? w1 : tile_of(a, (int)first));
    k.s1 = tiles_to(a, min(a.n_sink, end));
    k.skip = max(0, w0 - k.s1);
    k.n = min(k.s1, w1) + max(0, w1 - max(w0, k.s1));
  }
  return k;
}

struct PagedItem {
  int seq, begin, m, len, held;   // first packed row, new tokens, length, tokens that can lie in the cache
  int head_kv, first, rows;       // rows first .. first + rows - 1 of the sequence
  int part, parts, counter;       // which part of how many, and the row tile's counter
  int slot0, slot1, slot_step;    // where the first part, the second, and the others behind it lie in the workspace
  int t0, t1;                     // its key tiles
  KeyTiles keys;
  __device__ __forceinline__ int slot(int u) const { return u == 0 ? slot0 : slot1 + (u - 1) * slot_step; }
};

// ---- over a wavefront, by data-parallel moves within its registers: inclusive sums, and totals that every lane (and the scalar unit) has
__device__ __forceinline__ int scan_sum(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);   // the lane 1, 2, 4, 8 before, within 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // lanes 15 and 47 to the 16 behind
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // lane 31 to the 32 behind
  return v;
}
__device__ __forceinline__ int total_sum(int v) { return __builtin_amdgcn_readlane(scan_sum(v), 63); }
template <class F> __device__ __forceinline__ float total_of(float v, float neutral, F f) {
  auto moved = [&](auto ctrl, auto rows, float x) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(neutral), __float_as_uint(x), decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
  };
  using std::integral_constant;
  v = f(v, moved(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{}, v));
  v = f(v, moved(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{}, v));
  v = f(v, moved(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{}, v));
  v = f(v, moved(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{}, v));
  v = f(v, moved(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{}, v));
  v = f(v, moved(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{}, v));
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}

// a lane's sequence: T row tiles, of which the first sees v0 key tiles (at least 1) and the last v1
struct SeqWork {
  int begin, m, len, T, v0, v1;
};
struct SeqWords {   // as they lie in memory
  int begin, end, len;
};
__device__ __forceinline__ SeqWords seq_words(const PagedAttnArgs& a, int s) {
  return s < a.n_seqs ? SeqWords{a.cu[s], a.cu[s + 1], a.lens[s]} : SeqWords{0, 0, 0};
}
template <int BM> __device__ __forceinline__ SeqWork seq_work(const PagedAttnArgs& a, const SeqWords& w) {
  SeqWork q = {0, 0, 0, 0, 1, 1};
  q.begin = min(max(w.begin, 0), a.n_q);
  q.m = min(max(w.end, q.begin), a.n_q) - q.begin;
  q.len = max(w.len, 0);
  if (q.m > 0) {
    q.T = (q.m * a.group + BM - 1) / BM;
    const int held = min(q.len, a.max_pages * a.page);
    q.v0 = max(1, key_tiles(a, q.m, q.len, held, 0, min(q.m, div_group(a, BM - 1) + 1) - 1).n);
    q.v1 = max(1, key_tiles(a, q.m, q.len, held, div_group(a, (q.T - 1) * BM), q.m - 1).n);
  }
  return q;
}
// f(the lane's sequence) for every 64 sequences, the next ones on their way meanwhile
template <int BM, class F> __device__ __forceinline__ void each_64(const PagedAttnArgs& a, F f) {
  const int lane = thread_id() & 63;
  SeqWords next = seq_words(a, lane);
#pragma unroll 1
  for (int s0 = 0; s0 < a.n_seqs; s0 += kWave) {
    const SeqWords now = next;
    if (s0 + kWave < a.n_seqs) next = seq_words(a, s0 + kWave + lane);
    f(seq_work<BM>(a, now));
  }
}

// how the work is shared out (uniform)
struct PagedWork {
  bool shares;
  int C, each, split_each;   // pieces: tiles of a part at most, pieces of a key head, those of them that are parts
  int line, share;           // shares: the line's length for one key head, and a workgroup's share
};

// 64 sequences that are looked at: the lane's, what it extends over, how many of its pieces are parts, and what the sequences before extend over
struct SeqBlock {
  int s0;   // the first of them; < 0: none yet
  SeqWork q;
  int extent, split, before, split_before;
};


// pieces of C tiles: a sequence's parts lie in layers.  Row tile r is in layer p < layers() if it sees more than p C tiles, and so has as many
// parts as layers that hold it; new tokens see more the later they are, so that layer p holds the row tiles from first_row(p) on
__device__ __forceinline__ int layers(const SeqWork& q, int C) { return (int)((unsigned)(max(q.v0, q.v1) + C - 1) / (unsigned)C); }
template <int BM> __device__ __forceinline__ int first_row(const PagedAttnArgs& a, const SeqWork& q, int C, int p) {
  if (!a.causal || p * C < q.v0) return 0;
  const int token = min(max(tile_start(a, p * C) - (q.len - q.m), 0), max(q.m - 1, 0));
  return min(token * a.group / BM, max(q.T - 1, 0));
}
template <int BM> __device__ __forceinline__ int pieces_of(const PagedAttnArgs& a, const SeqWork& q, int C) {
  const int S = layers(q, C), all = a.causal && q.T > 1 ? min(S, (int)((unsigned)(q.v0 + C - 1) / (unsigned)C)) : S;
  int n = all * q.T;
  for (int p = all; p < S; ++p) n += q.T - first_row<BM>(a, q, C, p);
  return n;
}

constexpr int kNear = 4;     // a share ends at a row tile's end, or at least this many tiles from it

template <int BM> __device__ __forceinline__ int line_at(const SeqWork& q, int r, int lead) {   // where row tile r of a sequence lies
  const double slope = q.T > 1 ? 0.5 * (double)(q.v1 - q.v0) / (double)(q.T - 1) : 0.0;
  return (int)floor((double)r * (double)(q.v0 + lead) + slope * (double)r * (double)(r - 1));
}

template <int BM> __device__ __forceinline__ void find_extent(const PagedAttnArgs& a, const PagedSchedule& sc, const PagedWork& p, SeqBlock& block) {
  block.extent = p.shares ? line_at<BM>(block.q, block.q.T, sc.lead) : pieces_of<BM>(a, block.q, p.C);
  block.split = !p.shares && layers(block.q, p.C) > 1 ? block.extent : 0;
}

template <int BM, bool kShares> __device__ __forceinline__ PagedWork find_work(const PagedAttnArgs& a, const PagedSchedule& sc, SeqBlock& block) {
  const int lane = thread_id() & 63;
  const auto add = [](float x, float y) { return x + y; };
  const auto larger = [](float x, float y) { return fmaxf(x, y); };
  float units = 0.0f, rows = 0.0f, longest = 1.0f;
  SeqWork q = {0, 0, 0, 0, 1, 1};
  each_64<BM>(a, [&](const SeqWork& of) {
    q = of;
    // from row tile to row tile what they see grows by their tokens until it is v1 (shrinks, where a window ends and nothing is causal)
    const float v0 = (float)q.v0, v1 = (float)q.v1, T = (float)q.T;
    const float grows = fminf(T, fabsf(v1 - v0) * (float)(kKeyTile * a.group) * (1.0f / BM));
    units += T * v1 + 0.5f * grows * (v0 - v1);
    rows += T;
    longest = fmaxf(longest, (float)(q.T > 0 ? max(q.v0, q.v1) : 1));
  });
  PagedWork p = {false, 0x3fffffff, 0, 0, 0, 1};
  block = SeqBlock{-1, q, 0, 0, 0, 0};
  if (sc.meets) {
    units = total_of(units, 0.0f, add);
    rows = total_of(rows, 0.0f, add);
    longest = total_of(longest, 0.0f, larger);
    const float heads = (float)a.heads_kv, n = units / longest * heads;
    const float S = lane < 32 ? (float)(lane + 1) : floorf(32.0f * __builtin_amdgcn_exp2f((float)(lane - 31) * (5.0f / 32.0f)));   // .. 1024
    const float x = n * S * (1.0f / sc.units), full = fminf(x, 1.0f);
    const bool alike = units > 0.98f * longest * rows || (!kShares && lane > 0);
    const bool once = kShares ? x <= 1.0f && rows * heads <= sc.units : x <= 1.0f;   // (those that stay have theirs from the beginning)
    const float rounds = once ? 1.0f : (alike ? ceilf(x) : x + (kShares ? 0.75f : 0.5f));
    const float work = kShares ? rounds * fmaxf(sc.tile_alone + 0.3f * sc.tile * full, sc.tile * full)
                               : rounds * sc.tile + (rounds - 2.0f * floorf(0.5f * rounds)) * (sc.tile_alone - sc.tile);
    float cost = longest / S * work + rounds * sc.start + (lane > 0 ? sc.meet + sc.join * S : 0.0f);
    if (lane > 0 && (n * S > (float)sc.groups || S > longest)) cost = INFINITY;
    const float best = -total_of(-cost, -INFINITY, larger);
    const int at = __ffsll(__ballot(cost == best)) - 1;
    const float s_best = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(S), at));
    if constexpr (kShares) {
    const float line = (units + rows * (float)sc.lead) * heads;
    const float by_shares = line * (1.0f / sc.units) * sc.tile + 2.0f * sc.start + sc.meet + 3.0f * sc.join;
    p.shares = line < 1e9f && line > (float)(sc.groups * (sc.lead + 3 * kNear)) && by_shares < best;
    }
    if (!p.shares && at > 0) p.C = (int)ceilf(longest / s_best);
  }
  p.C = __builtin_amdgcn_readfirstlane(p.C);
  p.shares = kShares && __builtin_amdgcn_readfirstlane((int)p.shares);
  for (bool once = true;; once = false) {
    p.each = p.split_each = p.line = 0;
    const auto count = [&](const SeqWork& of) {
      block.q = of;
      find_extent<BM>(a, sc, p, block);
      const int sum = total_sum(block.extent);
      p.line += p.shares ? sum : 0;
      p.each += p.shares ? 0 : sum;
      p.split_each += total_sum(block.split);
    };
    if (a.n_seqs > kWave) each_64<BM>(a, count);
    else count(q);   // (they stay)
    // more than there is room for, which an estimate may come to: nothing is cut
    if (p.shares || !once || (p.split_each * a.heads_kv <= 2 * sc.groups && (kShares || p.each * a.heads_kv <= (int)gridDim.x))) break;
    p.C = 0x3fffffff;
  }
  if (a.n_seqs <= kWave) block.s0 = 0;
  if (p.shares) p.share = max((int)(((long long)p.line * a.heads_kv + sc.groups - 1) / sc.groups), sc.lead + 3 * kNear);
  return p;
}

// What both ways have in common: the sequence that holds place y, and what precedes it.  The 64 sequences that are looked at stay: a workgroup's
// next item is among them or behind, but for another head's (2048 single tokens over 3 to 60 keys 1096 us when every item began at the first, then 618; by a wavefront each 332)
template <int BM> __device__ __forceinline__ bool find_seq(const PagedAttnArgs& a, const PagedSchedule& sc, const PagedWork& p, int y, SeqBlock& block,
                                                          SeqWork& q, int& seq, int& before, int& split_before) {
  const int lane = thread_id() & 63;
  if (block.s0 < 0 || y < block.before) {
    if (block.s0 != 0) {
      block.q = seq_work<BM>(a, seq_words(a, lane));
      find_extent<BM>(a, sc, p, block);
    }
    block.s0 = block.before = block.split_before = 0;
  }
  while (true) {
    const int upto = block.before + scan_sum(block.extent), split_upto = block.split_before + scan_sum(block.split);
    const unsigned long long owner = __ballot(y >= upto - block.extent && y < upto);
    if (owner) {
      const int src = __ffsll(owner) - 1;
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, src); };
      q = SeqWork{of(block.q.begin), of(block.q.m), of(block.q.len), of(block.q.T), of(block.q.v0), of(block.q.v1)};
      seq = block.s0 + src;
      before = of(upto - block.extent);
      split_before = of(split_upto - block.split);
      return true;
    }
    if (block.s0 + kWave >= a.n_seqs) return false;
    block.s0 += kWave;
    block.before = __builtin_amdgcn_readlane(upto, 63);
    block.split_before = __builtin_amdgcn_readlane(split_upto, 63);
    block.q = seq_work<BM>(a, seq_words(a, block.s0 + lane));
    find_extent<BM>(a, sc, p, block);
  }
}

template <int BM> __device__ __forceinline__ void set_rows(const PagedAttnArgs& a, const SeqWork& q, int seq, int r, PagedItem& it) {
  it.seq = seq;
  it.begin = q.begin;
  it.m = q.m;
  it.len = q.len;
  it.held = min(q.len, a.max_pages * a.page);
  it.first = r * BM;
  it.rows = min(BM, q.m * a.group - it.first);
  it.keys = key_tiles(a, q.m, q.len, it.held, div_group(a, it.first), div_group(a, it.first + it.rows - 1));
}

// pieces: the `item`-th
template <int BM> __device__ __forceinline__ bool find_piece(const PagedAttnArgs& a, const PagedSchedule& sc, const PagedWork& p, int item, SeqBlock& block,
                                                           PagedItem& it) {
  if (item >= p.each * a.heads_kv) return false;
  it.head_kv = (int)((unsigned)item / (unsigned)p.each);
  const int y = item - it.head_kv * p.each, lane = thread_id() & 63;
  SeqWork q;
  int seq, before, split_before;
  if (!find_seq<BM>(a, sc, p, y, block, q, seq, before, split_before)) return false;
  // within a sequence: layer, then rows, the last ones (which see most) first.  A row tile's parts have consecutive places in the workspace
  const int S = layers(q, p.C), idx = y - before;
  int back, at = 0;   // at: parts of the row tiles behind this one
  if (!a.causal || q.T == 1 || S == 1) {
    it.part = (int)((unsigned)idx / (unsigned)q.T);
    it.parts = S;
    back = idx - it.part * q.T;
    at = back * S;
  } else {
    int done = 0;
    back = it.part = it.parts = 0;
    for (int p0 = 0; p0 < S; p0 += kWave) {
      const int e = p0 + lane < S ? q.T - first_row<BM>(a, q, p.C, p0 + lane) : 0, upto = done + scan_sum(e);
      const unsigned long long owner = __ballot(idx >= upto - e && idx < upto);
      if (owner) {
        const int src = __ffsll(owner) - 1;
        it.part = p0 + src;
        back = idx - __builtin_amdgcn_readlane(upto - e, src);
        break;
      }
      done = __builtin_amdgcn_readlane(upto, 63);
    }
    for (int p0 = 0; p0 < S; p0 += kWave) {
      const int e = p0 + lane < S ? q.T - first_row<BM>(a, q, p.C, p0 + lane) : 0;
      it.parts += __popcll(__ballot(back < e));
      at += total_sum(min(back, e));
    }
  }
  set_rows<BM>(a, q, seq, q.T - 1 - back, it);
  it.counter = it.slot0 = it.head_kv * p.split_each + split_before + at;   // (meant where there are parts)
  it.slot1 = it.slot0 + 1;
  it.slot_step = 1;
  const int each = (int)((unsigned)it.keys.n / (unsigned)it.parts), more = it.keys.n - each * it.parts;   // the first `more` parts have one more
  it.t0 = each * it.part + min(it.part, more);
  it.t1 = it.t0 + each + (it.part < more ? 1 : 0);
  return true;
}

// shares: the part at place x of the line, if it is workgroup `wg`'s (parts of a row tile belong to consecutive ones); else, parts = 0.
// next: where the row tile ends
template <int BM> __device__ __forceinline__ bool find_part(const PagedAttnArgs& a, const PagedSchedule& sc, const PagedWork& p, int wg, int x, SeqBlock& block, PagedItem& it,
                                                           int& next) {
  it.head_kv = x / p.line;
  if (it.head_kv >= a.heads_kv) return false;
  const int y = x - it.head_kv * p.line, lane = thread_id() & 63;
  SeqWork q;
  int seq, before, split_before;
  if (!find_seq<BM>(a, sc, p, y, block, q, seq, before, split_before)) return false;
  // the row tile: the last one that starts at or before y
  int lo = 0, span = q.T;
  while (span > 1) {
    const int step = (span + kWave - 1) / kWave, r = lo + lane * step;
    const int found = __popcll(__ballot(lane * step < span && line_at<BM>(q, r, sc.lead) <= y - before)) - 1;
    lo += found * step;
    span = min(step, span - found * step);
  }
  const int from = x - y + before + __builtin_amdgcn_readfirstlane(line_at<BM>(q, lo, sc.lead));
  const int to = x - y + before + __builtin_amdgcn_readfirstlane(line_at<BM>(q, lo + 1, sc.lead));
  next = to;
  // the shares' ends g share that cut it: g = g0 .. g1
  // (one near its beginning, but before its end: the whole row tile is the next workgroup's, which begins inside it)
  const int g0 = (min(from + sc.lead + kNear, to) + p.share - 1) / p.share, g1 = (to - kNear) / p.share, cuts = max(0, g1 - g0 + 1);
  it.part = min(max(x / p.share - g0 + 1, 0), cuts);
  it.parts = cuts + 1;
  if (g0 - 1 + it.part != wg) {
    if (g0 - 1 + it.part > wg) return false;
    it.parts = 0;
    return true;
  }
  set_rows<BM>(a, q, seq, lo, it);
  it.counter = g0 - 1;
  it.slot0 = 2 * (g0 - 1) + 1;
  it.slot1 = 2 * g0;
  it.slot_step = 2;
  auto tile_at = [&](int at) {   // of the row tile's n, at a place of the line
    return (int)((double)max(0, at - from - sc.lead) * (double)it.keys.n / (double)max(1, to - from - sc.lead));
  };
  it.t0 = it.part == 0 ? 0 : tile_at((g0 + it.part - 1) * p.share);
  it.t1 = it.part == cuts ? it.keys.n : tile_at((g0 + it.part) * p.share);
  return true;
}

// the workgroup's items one after another: state, and a step to the next (false: there is none).  kStay: workgroups stay for more than one
// and may have shares; else workgroup ids go round the XCDs so that each takes one contiguous eighth of the pieces, which read the same keys
struct PagedCursor {
  PagedWork work;
  SeqBlock block;
  int at, end;
};
template <int BM, bool kStay> __device__ __forceinline__ PagedCursor first_item(const PagedAttnArgs& a, const PagedSchedule& sc) {
  PagedCursor c;
  c.work = find_work<BM, kStay>(a, sc, c.block);
  const int id = (int)blockIdx.x;
  if (!kStay) {   // (the grid is a multiple of eight, and has at least as many workgroups as there are pieces)
    const int per = (c.work.each * a.heads_kv + 7) / 8;
    c.at = (id & 7) * per + (id >> 3);
    c.end = (id >> 3) < per ? c.at + 1 : c.at;
  } else if (c.work.shares) {
    c.at = id * c.work.share;
    c.end = c.at + c.work.share;
  } else {
    c.at = id;
    c.end = 0x7fffffff;
  }
  return c;
}
template <int BM, bool kStay> __device__ __forceinline__ bool next_item(const PagedAttnArgs& a, const PagedSchedule& sc, PagedCursor& c, PagedItem& it) {
  if (!kStay || !c.work.shares) {
    if (c.at >= c.end || !find_piece<BM>(a, sc, c.work, c.at, c.block, it)) return false;
    c.at += (int)gridDim.x;
    return true;
  }
  while (c.at < c.end) {
    int next;
    if (!find_part<BM>(a, sc, c.work, blockIdx.x, c.at, c.block, it, next)) return false;
    const bool mine = it.parts > 0;
    c.at = mine && it.part < it.parts - 1 ? c.end : next;   // (a cut is the share's end)
    if (mine) return true;
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

// whether one of the item's entries is no page (uniform; every wavefront looks at all of them; tiles from multiples of 32 on)
__device__ __forceinline__ bool any_bad_page(const PagedAttnArgs& a, const PagedItem& it) {
  if (it.t1 <= it.t0 || it.held == 0) return false;
  const int32_t* row = a.table + (long long)it.seq * a.max_pages;
  bool bad = false;
  auto scan = [&](int t0, int t1) {   // tiles t0 .. t1 - 1
    const int last = div_page(a, min(kKeyTile * it.keys.tile(t1 - 1) + kKeyTile, it.held) - 1);
    for (int e = div_page(a, kKeyTile * it.keys.tile(t0)) + (thread_id() & 63); e <= last; e += kWave) bad = bad || !is_page(a, row[e]);
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
  const int tid = thread_id(), f = 8 * (tid % TPR), r0 = tid / TPR;
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
    const int x = it.first + row, token = div_group(a, x), head = it.head_kv * a.group + (x - token * a.group);
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
  const __amdgpu_buffer_rsrc_t parts = __builtin_amdgcn_make_buffer_rsrc(sc.parts, 0, 2 * sc.groups * (BM * (D + 2) * 4), 0x00020000);
  const int stats_at_byte = 2 * sc.groups * (BM * D * 4);
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
    const int to = row_byte(it.slot(it.part), row);
    __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(acc[0]), __float_as_uint(acc[1]), __float_as_uint(acc[2]), __float_as_uint(acc[3])}, parts, to, 0, kSc1);
    __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(acc[4]), __float_as_uint(acc[5]), __float_as_uint(acc[6]), __float_as_uint(acc[7])}, parts, to + 16, 0, kSc1);
    if (f == 0) __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(M), __float_as_uint(L)}, parts, stat_byte(it.slot(it.part), row), 0, kSc1);
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
  // ---- the last one.  Few rows leave threads over: G sets of threads then take every G-th part each and meet in LDS, in their order
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
          const int slot = it.slot(min(u0 + i * G, it.parts - 1));
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
