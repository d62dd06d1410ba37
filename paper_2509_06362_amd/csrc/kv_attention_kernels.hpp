// Attention over the pages of a key/value cache, for sequences' newest tokens.
//
// Rows of the products are pairs (query token, query head of one key head); an item is 16 such rows against a part
// of the keys they share a page list for: a part of the tokens that a group of sequences begins with, or of what a
// sequence has of its own.  Over the keys runs the softmax's maximum m and sum l with the output's sum o:
//   m' = max(m, max_t s_t),  l' = l 2^(m - m') + sum_t 2^(s_t - m'),  o' = o 2^(m - m') + sum_t 2^(s_t - m') v_t,
// s in units of log2.  Parts of a row are joined the same way.
//
// Both products are turned round, s^T = K q^T and o^T = V^T p^T, on 16 x 16 x 32 matrix instructions: a lane then
// holds for one row the scores of the very keys that it needs as operand of the second product, so weights never
// leave registers; for that a lane's key rows are taken in the order 8 (m / 4) + m % 4 and + 4.  Keys and values come
// from the pages to registers as operands, 16 bytes a lane, without shared memory.
//
// Roundings to fewer bits: the outputs, and the weights, to the queries' type, in which the second product's values are: 32-bit
// products go at a sixteenth of the rate, and a weight as the sum of two 16-bit numbers takes that product twice.  A weight is off by
// half a step (2^-8 of it in bf16, 2^-11 in fp16), the sum l is of the unrounded ones; outputs are 1.2 to 1.4 times as far from
// 64 bits as a 32-bit form's rounded once (160 sequences in bf16: 0.0023 for 0.0017).  All else is 32 bits.
// What bounds it: few rows the pages' bytes where there are many (96 ragged rows in 8 bits, 268 MB, 65 us and 3 to join them:
// 4.0 TB/s) and latency where there are not (one row of 8191 keys: 34 MB in 11 us, then 4 to join its 32 parts); tiles below.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/maaso_instance.h"
#include "element_types.hpp"
#include "kv_pages_kernels.hpp"
#include "page_walk.hpp"

namespace maaso {

constexpr float kLn2 = 0.693147180559945309f;
constexpr uint32_t kStreamRows = 16;  // most rows of an item that one wave's registers take; more are taken in tiles

struct AttentionArgs {
  const void* q;
  void* out;
  float* lse;
  uint64_t q_stride, out_stride;
  const char* k_pages;  // the layer's
  const char* v_pages;
  uint64_t page_stride;  // elements
  const float* k_scale;
  const float* v_scale;
  const int32_t* table;
  const int32_t* length;
  const int32_t* q_start;
  const int32_t* rows;
  const int32_t* group_start;
  const int32_t* shared;
  uint32_t n, n_tok, n_heads, n_kv_heads, group, n_groups;
  uint32_t n_pages, page_log2, n_rows, width;
  uint32_t max_q, max_len, most_shared;  // most_shared: the caller's bound, within max_len and a row's width
  uint32_t own_least, shared_chunk;    // keys of an own part at least, of a shared one; multiples of 64
  uint32_t own_parts, shared_parts;    // most parts of a row
  uint32_t own_tiles, shared_tiles;    // most tiles of kTileRows rows
  uint32_t tile_blocks, stream_blocks; // of the launch of tiles
  uint32_t tile_shared, stream_shared; // blocks, items that take shared parts; those behind them take own ones
  bool alone;                          // items of few rows: a wave each, not a block
  float scale_log2;
  // workspace, where a row has several parts
  float* part_o;   // [part][n_tok * n_heads][D]
  float* part_ml;  // [part][n_tok * n_heads][2]
  uint32_t* status;
};

// A value that all lanes of a wave have alike, as one.
__device__ inline uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }

// What a sequence or a group has of rows and keys, from the device's arrays; everything within its bounds.
struct SequenceSpan {
  uint32_t row, tok0, n_q, len;
  int32_t before;  // tokens that its row held before its queries, all of them (negative: it holds fewer than they are)
};

// (What does not depend on one another is asked for at once, good or not: each load that waits for another is most of a
// microsecond of a short item.)
__device__ inline SequenceSpan sequence_span(const AttentionArgs& a, uint32_t i) {
  const int32_t q0 = a.q_start[i], q1 = a.q_start[i + 1], row = a.rows ? a.rows[i] : (int32_t)i;
  const bool known = row >= 0 && (uint32_t)row < a.n_rows;
  const int32_t len = a.length[known ? row : 0];
  SequenceSpan s{0u, 0u, 0u, 0u, 0};
  if (q0 < 0 || q1 < q0 || (uint32_t)q1 > a.n_tok) { raise(a.status, MAASO_INST_BAD_BOUND); return s; }
  s.tok0 = (uint32_t)q0;
  s.n_q = (uint32_t)(q1 - q0);
  if (s.n_q > a.max_q) { raise(a.status, MAASO_INST_BAD_BOUND); s.n_q = a.max_q; }
  if (!known) { raise(a.status, MAASO_INST_BAD_ROW); return s; }
  s.row = (uint32_t)row;
  if (len < 0 || (uint64_t)len > (uint64_t)a.width << a.page_log2) { raise(a.status, MAASO_INST_BAD_ROW); return s; }
  s.len = (uint32_t)len;
  s.before = len - (q1 - q0);
  if (s.len > a.max_len) { raise(a.status, MAASO_INST_BAD_BOUND); s.len = a.max_len; }
  return s;
}

// Keys that query j of a span sees, by the sequence's own length and queries, also where a bound leaves some of them out.
__device__ inline uint32_t seen_keys(int32_t before, uint32_t len, uint32_t j) {
  const uint32_t limit = (uint32_t)before + j + 1u;
  return (int32_t)limit < 0 ? 0u : limit < len ? limit : len;
}

// Whether group g's sequences, and their queries, are a range.
__device__ inline bool group_good(const AttentionArgs& a, uint32_t g) {
  const int32_t f = a.group_start[g], e = a.group_start[g + 1];
  if (f >= 0 && e >= f && (uint32_t)e <= a.n) {
    const int32_t q0 = a.q_start[f], q1 = a.q_start[e];
    if (q0 >= 0 && q1 >= q0 && (uint32_t)q1 <= a.n_tok) return true;
  }
  raise(a.status, MAASO_INST_BAD_BOUND);
  return false;
}

// Tokens that sequence i begins with like its group, as far as the caller's bound and a row's width go; 0 outside every
// group.  All lanes of the wave have the same i: 64 groups are looked at in one go.
struct GroupLanes {
  int32_t first, end, shared;
};
__device__ inline GroupLanes groups_from(const AttentionArgs& a, uint32_t base) {
  const uint32_t lane = threadIdx.x & 63u, g = base + lane < a.n_groups ? base + lane : a.n_groups - 1u;
  return {a.group_start[g], a.group_start[g + 1u], a.shared[g]};
}
__device__ inline uint32_t shared_of(const AttentionArgs& a, uint32_t i, GroupLanes at) {
  uint32_t found = 0;
  for (uint32_t base = 0; base < a.n_groups; base += 64u) {
    if (base) at = groups_from(a, base);
    const uint64_t which = __ballot(at.first >= 0 && at.first <= (int32_t)i && at.end > (int32_t)i && (uint32_t)at.end <= a.n);
    if (which) {
      const int32_t keys = __shfl(at.shared, __builtin_ctzll(which));
      if (keys < 0 || (uint32_t)keys > a.most_shared) raise(a.status, MAASO_INST_BAD_BOUND);
      found = keys < 0 ? 0u : (uint32_t)keys < a.most_shared ? (uint32_t)keys : a.most_shared;
      break;
    }
  }
  return found;
}

// The sequence i of token t: the last one that begins at t or before (t may lie behind its end, or before the first: then it
// is of none).  Where each sequence may have its one token, the span at its own place is looked at first.
__device__ inline SequenceSpan sequence_of(const AttentionArgs& a, uint32_t t, uint32_t& i) {
  if (a.max_q == 1u && a.n_tok == a.n) {
    i = t;
    const SequenceSpan s = sequence_span(a, i);
    if (t - s.tok0 < s.n_q) return s;
  }
  uint32_t lo = 0, hi = a.n;
  while (hi - lo > 1u) {
    const uint32_t mid = (lo + hi) >> 1;
    if ((uint32_t)a.q_start[mid] <= t) lo = mid; else hi = mid;
  }
  i = lo;
  return sequence_span(a, i);
}

// Tile `tile` of `rows` rows, counted through the sequences (or groups) with more than kStreamRows rows: which one, and
// its first row there.  Taken by every lane of a wave alike.
__device__ inline bool find_tile(const AttentionArgs& a, bool groups, uint32_t rows, uint32_t tile, uint32_t& which, uint32_t& row0) {
  const uint32_t count = groups ? a.n_groups : a.n, lane = threadIdx.x & 63u;
  uint32_t before = 0;
  for (uint32_t base = 0; base < count; base += 64u) {
    const uint32_t i = base + lane;
    uint32_t tiles = 0;
    if (i < count) {
      const bool known = !groups || group_good(a, i);
      const int32_t q0 = known ? a.q_start[groups ? (uint32_t)a.group_start[i] : i] : 0;
      const int32_t q1 = known ? a.q_start[groups ? (uint32_t)a.group_start[i + 1u] : i + 1u] : 0;
      if (q0 < 0 || q1 < q0 || (uint32_t)q1 > a.n_tok) raise(a.status, MAASO_INST_BAD_BOUND);
      else if ((uint64_t)(uint32_t)(q1 - q0) * a.group > kStreamRows) tiles = (uint32_t)(((uint64_t)(uint32_t)(q1 - q0) * a.group + rows - 1u) / rows);
    }
    uint32_t sum = tiles;
    for (uint32_t d = 1; d < 64u; d <<= 1) {
      const uint32_t y = __shfl_up(sum, d);
      if (lane >= d) sum += y;
    }
    const uint64_t behind = __ballot(before + sum > tile);
    if (behind) {
      const int at = __builtin_ctzll(behind);
      which = base + (uint32_t)at;
      row0 = (tile - before - (__shfl(sum, at) - __shfl(tiles, at))) * rows;
      return true;
    }
    before += __shfl(sum, 63);
  }
  return false;
}

// An item's rows and keys.
struct ItemKeys {
  uint32_t tok0, n_rows, begin, end, page_row, len;
  int32_t before;
  bool alone;  // its rows have no other part: their results are written as they are, not joined
};

// The end of an item's keys [begin, end), begin < end, as far as its page list holds pages: a bad entry is not followed, what
// lies behind it in the item is left out.  All lanes of the wave have the same item; `entries` becomes the list's first 64
// entries from begin's page on, a lane each, from a bad one on 0.
__device__ inline uint32_t held_end(const AttentionArgs& a, const int32_t* list, uint32_t begin, uint32_t end, int32_t& entries) {
  const uint32_t first = begin >> a.page_log2, last = (end - 1u) >> a.page_log2, lane = threadIdx.x & 63u;
  for (uint32_t page0 = first; page0 <= last; page0 += 64u) {
    const int32_t page = page0 + lane <= last ? list[page0 + lane] : 0;
    const uint64_t bad = __ballot(page < 0 || (uint32_t)page >= a.n_pages);
    if (page0 == first) entries = kept_entry(page, bad, lane);
    if (bad) {
      raise(a.status, MAASO_INST_BAD_PAGE);
      return end_before(page0, (uint32_t)__builtin_ctzll(bad), a.page_log2, begin);
    }
  }
  return end;
}

// Parts of a row: those of its group's keys, those of the sequence's own.  The own keys are cut into as many equal parts,
// of a multiple of 64 keys, as there are at most, but into none below own_least keys.
struct RowParts {
  uint32_t n_shared, n_own, own_chunk;
};
__device__ inline RowParts row_parts(const AttentionArgs& a, uint32_t len, uint32_t shared) {
  RowParts p{(shared + a.shared_chunk - 1u) / a.shared_chunk, 0u, a.own_least};
  if (len > shared) {
    const uint32_t own = len - shared, most = (own + a.own_least - 1u) / a.own_least, parts = most < a.own_parts ? most : a.own_parts;
    p.own_chunk = ((own + parts - 1u) / parts + 63u) & ~63u;
    p.n_own = (own + p.own_chunk - 1u) / p.own_chunk;
  }
  return p;
}

// False where there is nothing to do for part `part` of sequence or group `which` from row row0 on.
__device__ inline bool item_keys(const AttentionArgs& a, bool is_shared, uint32_t which, uint32_t part, uint32_t row0, ItemKeys& k) {
  if (is_shared) {
    const uint32_t f = (uint32_t)a.group_start[which], e = (uint32_t)a.group_start[which + 1];  // (group_good has seen them)
    const int32_t keys = a.shared[which];
    const SequenceSpan lead = sequence_span(a, f < a.n ? f : 0u);
    k.tok0 = (uint32_t)a.q_start[f];
    k.n_rows = ((uint32_t)a.q_start[e] - k.tok0) * a.group;
    k.page_row = lead.row;
    const uint32_t all = keys < 0 ? 0u : (uint32_t)keys < a.most_shared ? (uint32_t)keys : a.most_shared;
    if (keys < 0 || (uint32_t)keys > a.most_shared || all > lead.len) raise(a.status, MAASO_INST_BAD_BOUND);
    k.alone = false;
    k.begin = part * a.shared_chunk;
    k.end = k.begin + a.shared_chunk < all ? k.begin + a.shared_chunk : all;
    // (each part of `all` is written, whatever the first row holds of it: the join counts them)
    if (k.begin >= k.end || k.n_rows == 0u) return false;
    k.end = k.end < lead.len ? k.end : lead.len;
    k.end = k.end < k.begin ? k.begin : k.end;
    return row0 < k.n_rows;
  } else {
    GroupLanes groups{-1, -1, 0};
    if (a.n_groups) groups = groups_from(a, 0u);
    const SequenceSpan s = sequence_span(a, which);
    k.tok0 = s.tok0;
    k.before = s.before;
    k.len = s.len;
    k.n_rows = s.n_q * a.group;
    k.page_row = s.row;
    const uint32_t shared = shared_of(a, which, groups);
    const RowParts parts = row_parts(a, s.len, shared);
    k.alone = parts.n_shared + parts.n_own <= 1u && parts.n_shared == 0u;
    const uint64_t b = (uint64_t)shared + (uint64_t)part * parts.own_chunk;
    k.begin = b < s.len ? (uint32_t)b : s.len;
    k.end = s.len - k.begin < parts.own_chunk ? s.len : k.begin + parts.own_chunk;
  }
  // Without keys there is nothing to join; rows without any are written all the same, by the first part.
  if (k.begin >= k.end) {
    if (!k.alone || part) return false;
    k.end = k.begin;
  }
  return row0 < k.n_rows;
}

// Keys that token tok of the item sees.
__device__ inline uint32_t row_limit(const AttentionArgs& a, bool is_shared, const ItemKeys& k, uint32_t tok) {
  if (!is_shared) return seen_keys(k.before, k.len, tok - k.tok0);
  uint32_t i;
  const SequenceSpan s = sequence_of(a, tok, i);
  return seen_keys(s.before, s.len, tok - s.tok0);
}

// Eight neighbouring elements as they lie in a page: widened to operands; those of [from, to) kept and the others made zeros,
// whatever they hold (by their bits); whether one is an infinity or NaN.
template <typename T, typename C> struct KeyLoad;
template <typename T> struct KeyLoad<T, T> {
  using raw = typename Vec<T>::x8;
  using bits = u32x4;
  static __device__ inline typename Vec<T>::x8 wide(raw r) { return r; }
  static __device__ inline bits kept(uint32_t from, uint32_t to) {
    bits m;
#pragma unroll
    for (uint32_t k = 0; k < 4u; ++k)
      m[k] = (2u * k >= from && 2u * k < to ? 0xffffu : 0u) | (2u * k + 1u >= from && 2u * k + 1u < to ? 0xffff0000u : 0u);
    return m;
  }
  static __device__ inline bool odd(bits b) {
    constexpr uint32_t kTop = sizeof(T) == 2 && __is_same(T, __bf16) ? 0x7f80u : 0x7c00u;
    bool odd = false;
#pragma unroll
    for (int k = 0; k < 4; ++k) odd = odd || (b[k] & kTop) == kTop || (b[k] >> 16 & kTop) == kTop;
    return odd;
  }
};
template <typename T> struct KeyLoad<T, E4m3> {
  using raw = u32x2;
  using bits = u32x2;
  static __device__ inline typename Vec<T>::x8 wide(raw r) { return widen8<T>(r); }
  static __device__ inline bits kept(uint32_t from, uint32_t to) {
    bits m;
#pragma unroll
    for (uint32_t w = 0; w < 2u; ++w) {
      m[w] = 0u;
#pragma unroll
      for (uint32_t k = 0; k < 4u; ++k)
        if (w * 4u + k >= from && w * 4u + k < to) m[w] |= 0xffu << (8u * k);
    }
    return m;
  }
  // (seven ones: the one value that is none)
  static __device__ inline bool odd(bits b) { return (((b[0] & 0x7f7f7f7fu) + 0x01010101u) | ((b[1] & 0x7f7f7f7fu) + 0x01010101u)) & 0x80808080u; }
};

template <typename V> __device__ inline bool finite16(V v) {
  bool f = true;
#pragma unroll
  for (int k = 0; k < 8; ++k) f = f && __builtin_isfinite((float)v[k]);
  return f;
}

// One tile of rows against this wave's steps of 32 keys.  First the steps that not all rows see in full, if there are any,
// then the others, of which with heads of 64 the next one's keys and values are asked for before this one's are multiplied.
template <typename T, typename C, int D>
struct StreamTile {
  using X8 = typename Vec<T>::x8;
  using L = KeyLoad<T, C>;
  struct Step {
    typename L::raw k0[D / 32], k1[D / 32], v[D / 16];
  };
  X8 q[D / 32];
  f32x4 o[D / 16];
  float m, l, scale;
  const C* kp;  // the head's
  const C* vp;
  const int32_t* list;
  uint32_t begin, end, limit, lowest;  // keys of the item; those that this lane's row sees; the least that any row sees
  int32_t entries;                     // the page list's, 64 of them from entry0 on, a lane each
  uint32_t entry0;

  __device__ inline void clear() {
#pragma unroll
    for (int d = 0; d < D / 16; ++d) o[d] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    m = -INFINITY;
    l = 0.0f;
  }

  // The keys from `base` on, a multiple of 32: two pages at most.
  __device__ inline void ask(const AttentionArgs& a, Step& s, uint32_t base) {
    const uint32_t lane = threadIdx.x & 63u, col = lane & 15u, g = lane >> 4, per = 1u << a.page_log2;
    const uint32_t page_at = base >> a.page_log2;
    if (beyond_entries(page_at, entry0)) {
      entry0 = page_at;
      const uint32_t page = entry0 + lane;  // (a step may begin a page before the item, where held_end() has not looked)
      entries = page_of_item(page, begin, end, a.page_log2) ? list[page] : 0;
    }
    const uint32_t at = uniform(page_at - entry0);
    const uint32_t page0 = (uint32_t)__builtin_amdgcn_readlane(entries, (int)at);
    const uint32_t page1 = (uint32_t)__builtin_amdgcn_readlane(entries, (int)second_entry(at, a.page_log2));
    const uint32_t kpage = col >> 3 ? page1 : page0, vpage = g >> 1 ? page1 : page0;
    const uint32_t row = (base + 8u * (col >> 2) + (col & 3u)) & (per - 1u);
    const C* kr = kp + (uint64_t)kpage * a.page_stride + row * (uint32_t)D + g * 8u;
    const __attribute__((address_space(1))) C* vr = (const __attribute__((address_space(1))) C*)vp + (uint64_t)vpage * a.page_stride + ((base + 8u * g) & (per - 1u)) + (col << a.page_log2);
#pragma unroll
    for (int t = 0; t < D / 32; ++t) {
      s.k0[t] = *reinterpret_cast<const typename L::raw*>(kr + t * 32);
      s.k1[t] = *reinterpret_cast<const typename L::raw*>(kr + 4 * D + t * 32);
    }
#pragma unroll
    for (int d = 0; d < D / 16; ++d) {
      s.v[d] = *reinterpret_cast<const __attribute__((address_space(1))) typename L::raw*>(vr);
      vr += 16u << a.page_log2;
      asm volatile("" : "+v"(vr));  // (one address, moved on; it is named global, which the compiler cannot see behind this)
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  __device__ inline void scores(const Step& s, float (&x)[8]) const {
    f32x4 s0 = {0.0f, 0.0f, 0.0f, 0.0f}, s1 = s0;
#pragma unroll
    for (int t = 0; t < D / 32; ++t) {
      s0 = mfma_16x16x32(L::wide(s.k0[t]), q[t], s0);
      s1 = mfma_16x16x32(L::wide(s.k1[t]), q[t], s1);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[k] = s0[k] * scale;
      x[k + 4] = s1[k] * scale;
    }
  }

  __device__ inline X8 weights(const float (&x)[8]) {
    float top = x[0];
#pragma unroll
    for (int k = 1; k < 8; ++k) top = fmaxf(top, x[k]);
    // The maximum follows only where it has grown by more than 8 (weights up to 256 are as exact as up to 1); else the sums
    // need not be scaled, and the lanes of a row need not hear of each other.
    if (__any(top > m + 8.0f)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float now = fmaxf(m, top), turn = __builtin_amdgcn_exp2f(m - (now == -INFINITY ? 0.0f : now));
      l *= turn;
      m = now;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) o[d] = o[d] * turn;
    }
    const float zero = m == -INFINITY ? 0.0f : m;
    float p[8], sum = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      p[k] = __builtin_amdgcn_exp2f(x[k] - zero);
      sum += p[k];
    }
    l += sum;
    return narrow8<T>(p);
  }

  // Keys that every row sees.
  __device__ inline void take(const Step& s) {
    float x[8];
    scores(s, x);
    const X8 w = weights(x);
#pragma unroll
    for (int d = 0; d < D / 16; ++d) o[d] = mfma_16x16x32(L::wide(s.v[d]), w, o[d]);
  }

  // Keys of which some are not of the item, or not seen by all rows.
  __device__ inline void take_some(Step& s, uint32_t base) {
    const uint32_t lane = threadIdx.x & 63u, col = lane & 15u, key8 = base + 8u * (lane >> 4);
    float x[8];
    scores(s, x);
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (key8 + k < begin || key8 + k >= end || key8 + k >= limit) x[k] = -INFINITY;
    const X8 w = weights(x);
    // Values of keys that no row sees are taken as zeros, whatever their place holds; where one that some rows may see and others
    // not is not finite, row by row.
    auto keep = [&](uint32_t sees) {
      const uint32_t from = begin < key8 ? 0u : begin - key8, to = sees > key8 ? sees - key8 : 0u;
      return L::kept(from, to);
    };
    const typename L::bits held = keep(end);
    bool odd = false;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) {
      const typename L::bits b = __builtin_bit_cast(typename L::bits, s.v[d]) & held;
      s.v[d] = __builtin_bit_cast(typename L::raw, b);
      odd = odd || L::odd(b);
    }
    if (!__any(odd)) {
#pragma unroll
      for (int d = 0; d < D / 16; ++d) o[d] = mfma_16x16x32(L::wide(s.v[d]), w, o[d]);
      return;
    }
#pragma unroll 1
    for (int r = 0; r < 16; ++r) {
      const uint32_t most = __shfl(limit, r);
      const typename L::bits seen = keep(most < end ? most : end);
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
        typename L::bits b = __builtin_bit_cast(typename L::bits, s.v[d]) & seen;
        asm volatile("" : "+v"(b));  // (one after the other: registers are few)
        const f32x4 t = mfma_16x16x32(L::wide(__builtin_bit_cast(typename L::raw, b)), w, o[d]);
        if (col == (uint32_t)r) o[d] = t;
        asm volatile("" : "+v"(o[d]));
      }
    }
  }

  // This wave's steps, one of every kSplit.
  template <uint32_t kSplit>
  __device__ inline void run(const AttentionArgs& a, uint32_t wave) {
    constexpr uint32_t kStride = 32u * kSplit;
    end = uniform(held_end(a, list, begin, end, entries));
    entry0 = begin >> a.page_log2;
    if (begin >= end) return;
    const uint32_t whole0 = (begin + 31u) & ~31u, seen = lowest < end ? lowest : end;
    const uint32_t whole1 = (seen & ~31u) > whole0 ? seen & ~31u : whole0;  // [whole0, whole1): steps that all rows see in full
    const uint32_t before = begin < whole0 && begin / 32u < (end + 31u) / 32u ? 1u : 0u;
    const uint32_t others = before + (end > whole1 ? (end - whole1 + 31u) / 32u : 0u);
    // (the last waves have the fewest whole steps)
#pragma unroll 1
    for (uint32_t n = kSplit - 1u - wave; n < others; n += kSplit) {
      const uint32_t at = n < before ? begin & ~31u : whole1 + (n - before) * 32u;
      Step s;
      ask(a, s, at);
      take_some(s, at);
    }
    uint32_t base = whole0 + wave * 32u;
    if constexpr (D >= 128) {  // (two of them would be a third of the registers, or more)
#pragma unroll 1
      for (; base < whole1; base += kStride) {
        Step s;
        ask(a, s, base);
        take(s);
      }
      return;
    }
    if (base >= whole1) return;
    Step s0, s1;
    ask(a, s0, base);
    for (;;) {
      base += kStride;
      if (base >= whole1) { take(s0); return; }
      ask(a, s1, base);
      take(s0);
      base += kStride;
      if (base >= whole1) { take(s1); return; }
      ask(a, s0, base);
      take(s1);
    }
  }
};

// Items of few rows.  kSplit 1: a wave takes an item, alone; kSplit 4: the four waves of a block share an item's keys and join
// in shared memory, for when there are few items and the parts of a row would be many.
template <typename T, int D> struct StreamJoin {
  float o[4][16][D + 4];
  float m[4][16], l[4][16];
};

template <typename T, typename C, int D, int kSplit>
__device__ inline void stream_block(const AttentionArgs& a, uint32_t block, StreamJoin<T, D>* meet) {
  using X8 = typename Vec<T>::x8;
  const uint32_t lane = threadIdx.x & 63u, wave = uniform(threadIdx.x >> 6), col = lane & 15u, g = lane >> 4;
  // item -> (part, head, sequence or group)
  uint32_t id = kSplit == 1 ? block * 4u + wave : block;
  const bool is_shared = id < a.stream_shared;
  if (!is_shared) id -= a.stream_shared;
  const uint32_t head = id % a.n_kv_heads;
  id /= a.n_kv_heads;
  const uint32_t count = is_shared ? a.n_groups : a.n, which = id % count, part = id / count;
  if (!is_shared && part >= a.own_parts) return;  // (the last block's waves)
  if (is_shared && !group_good(a, which)) return;
  ItemKeys keys;
  if (!item_keys(a, is_shared, which, part, 0u, keys) || keys.n_rows > kStreamRows) return;
  const uint32_t n_rows = keys.n_rows;
  const bool real = col < n_rows;
  const uint32_t tok = keys.tok0 + (real ? col : 0u) / a.group, h = head * a.group + (real ? col : 0u) % a.group;
  const uint32_t limit = row_limit(a, is_shared, keys, tok);
  uint32_t lowest = limit, highest = limit;
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) {
    const uint32_t x = __shfl_xor(lowest, d), y = __shfl_xor(highest, d);
    lowest = x < lowest ? x : lowest;
    highest = y > highest ? y : highest;
  }
  StreamTile<T, C, D> st;
  const T* qp = static_cast<const T*>(a.q) + (uint64_t)tok * a.q_stride + (uint64_t)h * D + g * 8u;
#pragma unroll
  for (int s = 0; s < D / 32; ++s) st.q[s] = *reinterpret_cast<const X8*>(qp + s * 32);
  st.clear();
  st.kp = reinterpret_cast<const C*>(a.k_pages) + ((uint64_t)head << a.page_log2) * D;
  st.vp = reinterpret_cast<const C*>(a.v_pages) + ((uint64_t)head << a.page_log2) * D;
  st.list = a.table + (uint64_t)keys.page_row * a.width;
  st.begin = uniform(keys.begin);
  st.end = uniform(keys.end < highest ? keys.end : highest);
  st.limit = limit;
  st.lowest = uniform(lowest);
  st.scale = a.scale_log2 * (sizeof(C) == 1 && a.k_scale ? a.k_scale[head] : 1.0f);
  if (st.begin < st.end) st.template run<kSplit>(a, kSplit == 1 ? 0u : wave);
  float l = st.l;
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  const float vs = sizeof(C) == 1 && a.v_scale ? a.v_scale[head] : 1.0f;
  const uint64_t slot0 = (uint64_t)(is_shared ? part : a.shared_parts + part) * a.n_tok * a.n_heads;
  if constexpr (kSplit == 1) {
    if (!real) return;
    const uint64_t row = (uint64_t)tok * a.n_heads + h;
    if (keys.alone) {
      const float by = l == 0.0f ? 0.0f : vs / l;
      T* to = static_cast<T*>(a.out) + (uint64_t)tok * a.out_stride + (uint64_t)h * D + 4u * g;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
        const f32x4 y = l == 0.0f ? (f32x4){0.0f, 0.0f, 0.0f, 0.0f} : st.o[d] * by;
        typename Vec<T>::x2* at = reinterpret_cast<typename Vec<T>::x2*>(to + d * 16);
        at[0] = narrow2<T>(y[0], y[1]);
        at[1] = narrow2<T>(y[2], y[3]);
      }
      if (a.lse && g == 0u) a.lse[row] = l == 0.0f ? -INFINITY : (st.m + log2f(l)) * kLn2;
    } else {
      float* to = a.part_o + (slot0 + row) * D + 4u * g;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) *reinterpret_cast<f32x4*>(to + d * 16) = st.o[d];
      if (g == 0u) *reinterpret_cast<f32x2*>(a.part_ml + (slot0 + row) * 2) = (f32x2){st.m, l};
    }
  } else {
    // join the waves
    auto &so = meet->o;
    auto &sm = meet->m, &sl = meet->l;
    if (g == 0) { sm[wave][col] = st.m; sl[wave][col] = l; }
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, sm[w][col]);
    const float turn = __builtin_amdgcn_exp2f(st.m - (top == -INFINITY ? 0.0f : top));
#pragma unroll
    for (int d = 0; d < D / 16; ++d) *reinterpret_cast<f32x4*>(&so[wave][col][d * 16 + 4 * g]) = st.o[d] * turn;
    __syncthreads();
    const uint32_t orow = threadIdx.x >> 4, at = (threadIdx.x & 15u) * (D / 16);
    if (orow >= n_rows) return;
    float mm = -INFINITY, ll = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) mm = fmaxf(mm, sm[w][orow]);
    const float zero = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
    for (int w = 0; w < 4; ++w) ll += sl[w][orow] * __builtin_amdgcn_exp2f(sm[w][orow] - zero);
    float acc[D / 16];
#pragma unroll
    for (int k = 0; k < D / 16; ++k) acc[k] = (so[0][orow][at + k] + so[1][orow][at + k]) + (so[2][orow][at + k] + so[3][orow][at + k]);
    const uint32_t otok = keys.tok0 + orow / a.group, oh = head * a.group + orow % a.group;
    const uint64_t row = (uint64_t)otok * a.n_heads + oh;
    if (keys.alone) {
      const float by = ll == 0.0f ? 0.0f : vs / ll;
      T* to = static_cast<T*>(a.out) + (uint64_t)otok * a.out_stride + (uint64_t)oh * D + at;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) to[k] = (T)(ll == 0.0f ? 0.0f : acc[k] * by);
      if (a.lse && at == 0) a.lse[row] = ll == 0.0f ? -INFINITY : (mm + log2f(ll)) * kLn2;
    } else {
#pragma unroll
      for (int k = 0; k < D / 16; ++k) a.part_o[(slot0 + row) * D + at + k] = acc[k];
      if (at == 0) *reinterpret_cast<f32x2*>(a.part_ml + (slot0 + row) * 2) = (f32x2){mm, ll};
    }
  }
}

// Blocks to a compute unit, by the registers they need: with heads of 128 three of one step each beat two of two steps (160
// short sequences behind a shared beginning 110 to 105 us), with heads of 64 two steps have room beside three others.
template <typename T, typename C, int D, int kSplit>
__global__ void __launch_bounds__(256, D == 256 ? 2 : 3) attention_stream_kernel(AttentionArgs a) {
  if constexpr (kSplit == 1) {
    stream_block<T, C, D, 1>(a, blockIdx.x, nullptr);
  } else {
    __shared__ StreamJoin<T, D> meet;
    stream_block<T, C, D, kSplit>(a, blockIdx.x, &meet);
  }
}

// Many rows: a block of four waves takes 128 rows, 32 a wave, and steps through the keys kKeys at a time.  Keys and
// values of a step are brought to shared memory once for all four waves, the next step's while this one's are
// multiplied (asynchronously from the pages, without passing registers; from a cache of 8 bits through registers, where they
// are widened).  The products are the turned ones again, on 32 x 32 x 16 instructions, whose result holds key 8 j + 4 h + i
// of its 32 in element 4 j + i of lane half h: key rows are read in the order that makes those eight neighbours.
//
// 620 to 650 TFLOP/s where a large product reaches 1204: in a step the products, the reads of shared memory, the exponentials and the
// next step's addresses take turns and none fills it (without exponentials 4 % less time, with a quarter of the reads 8 %, without loads
// 13 %; no bank conflicts), and of 9 prompts' blocks the last round on the card is a fifth full.
//
// Rows lie in shared memory as they come from the pages, but for their 16-byte pieces, of which piece c lies at place
// c ^ f(row): the sixteen lanes that are served at once then meet sixteen different places of the 256 bytes of a cycle.
constexpr uint32_t kTileRows = 128;

template <typename T, typename C, int D, int kKeys>
struct RowTile {
  using X8 = typename Vec<T>::x8;
  static constexpr uint32_t kKeyBytes = kKeys * D * 2, kBuffer = 2 * kKeyBytes;
  static constexpr uint32_t kKeyRows = 1024 / (D * 2), kValueRows = 1024 / (kKeys * 2);  // rows that a wave brings at once
  static constexpr uint32_t kKeyLoads = kKeys / 4 / kKeyRows, kValueLoads = D / 4 / kValueRows;
  static constexpr bool kDirect = sizeof(C) == 2;  // from the pages to shared memory as they are

  char* lds;
  uint32_t lds_base;  // its address in shared memory
  uint32_t lane, wave, half, col, per;
  uint32_t key_at, value_at;  // where this lane reads operands, the place's lowest bits crossed with f
  const C* kp;
  const C* vp;
  uint64_t page_stride;
  uint32_t page_log2;
  u32x2 raw_k[kDirect ? 1 : kKeyLoads], raw_v[kDirect ? 1 : kValueLoads];

  // By the lane that reads the row (key rows are read in another order, see key()): its low four bits; the next three
  // where two rows of eight places fill 256 bytes, two where four rows of four do.
  static __device__ inline uint32_t by_lane(uint32_t c, uint32_t places) {
    return places >= 16u ? c & 15u : places == 8u ? c >> 1 & 7u : c >> 2 & 3u;
  }
  static __device__ inline uint32_t fk(uint32_t row) {
    return by_lane((row & 3u) | (row >> 3 & 1u) << 2 | (row >> 2 & 1u) << 3, D / 8);
  }
  static __device__ inline uint32_t fv(uint32_t row) { return by_lane(row, kKeys / 8); }

  // 16 bytes a lane from the pages to 1024 bytes of shared memory from `to` on.  Written out, because the compiler would
  // have every later read of shared memory wait for it; the loop waits itself, once a step.  (m0 is named as changed, so that
  // none of the compiler's own uses of it, from its setting on, has this between; that it warns of, as of any reserved register.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  __device__ inline void async16(const void* from, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_base + to), "v"(from) : "memory", "m0");
  }
#pragma clang diagnostic pop

  // Brings keys and values from `base` on; ids: lane c < kKeys / 8 (and every kKeys / 8 after it) holds the page of keys base + 8 c.
  __device__ inline void bring(uint32_t buffer, uint32_t base, int32_t ids) {
    constexpr uint32_t kChunks = D / 8, kPieces = kKeys / 8;
    const uint32_t row0 = wave * (kKeys / 4);
    const uint32_t kpage = (uint32_t)__builtin_amdgcn_readlane(ids, (int)__builtin_amdgcn_readfirstlane((int)(row0 / 8u)));
    const C* kb = kp + (uint64_t)kpage * page_stride;
#pragma unroll
    for (uint32_t it = 0; it < kKeyLoads; ++it) {
      const uint32_t row = row0 + it * kKeyRows + lane / kChunks, place = lane % kChunks;
      const C* from = kb + ((base + row) & (per - 1u)) * (uint32_t)D + (place ^ fk(row)) * 8u;
      if constexpr (kDirect) async16(from, buffer * kBuffer + (row0 + it * kKeyRows) * (D * 2));
      else raw_k[it] = *reinterpret_cast<const u32x2*>(from);
    }
    // (f of a value row has a bit that changes with `it`: two pieces, by turns)
    const C* vb[2];
#pragma unroll
    for (uint32_t turn = 0; turn < 2u; ++turn) {
      const uint32_t piece = lane % kPieces ^ fv(turn * kValueRows + lane / kPieces);
      const uint32_t vpage = (uint32_t)__shfl(ids, (int)piece);
      vb[turn] = vp + (uint64_t)vpage * page_stride + ((base + 8u * piece) & (per - 1u));
    }
#pragma unroll
    for (uint32_t it = 0; it < kValueLoads; ++it) {
      const uint32_t row = wave * (D / 4) + it * kValueRows + lane / kPieces;
      const C* from = vb[it & 1u] + ((uint64_t)row << page_log2);
      if constexpr (kDirect) async16(from, buffer * kBuffer + kKeyBytes + (wave * (D / 4) + it * kValueRows) * (kKeys * 2));
      else raw_v[it] = *reinterpret_cast<const u32x2*>(from);
    }
  }

  // What bring() has left in registers goes to shared memory.
  __device__ inline void settle(uint32_t buffer) {
    if constexpr (kDirect) {
      (void)buffer;
    } else {
      char* to = lds + buffer * kBuffer + lane * 16u;
#pragma unroll
      for (uint32_t it = 0; it < kKeyLoads; ++it)
        *reinterpret_cast<X8*>(to + (wave * (kKeys / 4) + it * kKeyRows) * (D * 2)) = widen8<T>(raw_k[it]);
#pragma unroll
      for (uint32_t it = 0; it < kValueLoads; ++it)
        *reinterpret_cast<X8*>(to + kKeyBytes + (wave * (D / 4) + it * kValueRows) * (kKeys * 2)) = widen8<T>(raw_v[it]);
    }
  }

  __device__ inline void aim() {
    const uint32_t row = 16u * (col >> 4) + 8u * (col >> 2 & 1u) + 4u * (col >> 3 & 1u) + (col & 3u);
    key_at = row * (D * 2) + ((half ^ fk(row)) << 4);
    value_at = kKeyBytes + col * (kKeys * 2) + ((half ^ fv(col)) << 4);
  }
  // (piece 2 s + half: bits above the first cross with what aim() has left there)
  __device__ inline X8 key(uint32_t buffer, uint32_t block, uint32_t s) const {
    constexpr uint32_t kCrossed = D == 64 ? 4u : 8u;
    return *reinterpret_cast<const X8*>(lds + ((buffer * kBuffer + key_at) ^ (s % kCrossed << 5)) + block * 32u * (D * 2) + s / kCrossed * 256u);
  }
  __device__ inline X8 value(uint32_t buffer, uint32_t d, uint32_t t) const {
    return *reinterpret_cast<const X8*>(lds + ((buffer * kBuffer + value_at) ^ (t << 5)) + d * 32u * (kKeys * 2));
  }
};

// Asks the scheduler for kProducts products, each with its operand read kAhead products before it.
template <int kProducts>
__device__ inline void feed() {
  constexpr int kAhead = kProducts < 6 ? kProducts : 6;
  __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);  // reads of shared memory
#pragma unroll
  for (int k = kAhead; k < kProducts; ++k) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a product
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
}

template <typename T, typename C, int D, int kKeys>
__device__ inline void tile_block(const AttentionArgs& a, uint32_t block, char* lds, uint32_t* lowest_of) {
  using X8 = typename Vec<T>::x8;
  using Tile = RowTile<T, C, D, kKeys>;
  constexpr int kBlocks = kKeys / 32, kSteps = kKeys / 16;
  const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31u, half = lane >> 5;
  const bool is_shared = block < a.tile_shared;
  uint32_t id = is_shared ? block : block - a.tile_shared;
  const uint32_t head = id % a.n_kv_heads;
  id /= a.n_kv_heads;
  const uint32_t tiles = is_shared ? a.shared_tiles : a.own_tiles;
  uint32_t which, row0;
  const uint32_t part = id / tiles;
  if (!find_tile(a, is_shared, kTileRows, id % tiles, which, row0)) return;
  ItemKeys keys;
  if (!item_keys(a, is_shared, which, part, row0, keys)) return;
  // this lane's row
  const uint32_t r = row0 + wave * 32u + col;
  const bool real = r < keys.n_rows;
  const uint32_t tok = keys.tok0 + (real ? r : row0) / a.group, h = head * a.group + (real ? r : row0) % a.group;
  const uint32_t limit = real ? row_limit(a, is_shared, keys, tok) : 0u;
  uint32_t lowest = real ? limit : 0xffffffffu, highest = limit;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t x = __shfl_xor(lowest, d), y = __shfl_xor(highest, d);
    lowest = x < lowest ? x : lowest;
    highest = y > highest ? y : highest;
  }
  if (lane == 0) lowest_of[wave] = lowest;
  __syncthreads();
  const uint32_t low2 = lowest_of[0] < lowest_of[1] ? lowest_of[0] : lowest_of[1], low3 = lowest_of[2] < lowest_of[3] ? lowest_of[2] : lowest_of[3];
  const uint32_t block_lowest = low2 < low3 ? low2 : low3;
  // A sequence's rows see more with every token: what the block's last row sees is the end.
  const uint32_t begin = uniform(keys.begin);
  uint32_t end = keys.end;
  if (!is_shared) {
    const uint32_t last = row0 + kTileRows < keys.n_rows ? row0 + kTileRows - 1u : keys.n_rows - 1u;
    const uint32_t most = row_limit(a, false, keys, keys.tok0 + last / a.group);
    end = most < end ? most : end;
    end = end < begin ? begin : end;
  }
  const float scale0 = a.scale_log2 * (sizeof(C) == 1 && a.k_scale ? a.k_scale[head] : 1.0f);
  const float scale = scale0 == 0.0f ? 1.0f : fabsf(scale0);
  X8 q[D / 16];
  {
    // (a negative scale turns the queries' signs, a scale of zero makes them zero: so the largest score is the largest product)
    const T* qp = static_cast<const T*>(a.q) + (uint64_t)tok * a.q_stride + (uint64_t)h * D + half * 8u;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      q[s] = *reinterpret_cast<const X8*>(qp + s * 16);
      if (!(scale0 > 0.0f)) {
#pragma unroll
        for (int k = 0; k < 8; ++k) q[s][k] = scale0 == 0.0f ? (T)0.0f : -q[s][k];
      }
    }
  }
  f32x16 o[D / 32];
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.0f;
  float m = -INFINITY, l = 0.0f;

  Tile tile;
  tile.lds = lds;
  tile.lane = lane;
  tile.wave = wave;
  tile.half = half;
  tile.col = col;
  tile.lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  tile.aim();
  tile.per = 1u << a.page_log2;
  tile.page_log2 = a.page_log2;
  tile.page_stride = a.page_stride;
  tile.kp = reinterpret_cast<const C*>(a.k_pages) + ((uint64_t)head << a.page_log2) * D;
  tile.vp = reinterpret_cast<const C*>(a.v_pages) + ((uint64_t)head << a.page_log2) * D;
  const int32_t* list = a.table + (uint64_t)keys.page_row * a.width;
  int32_t held = 0;
  if (begin < end) {
    end = uniform(held_end(a, list, begin, end, held));
  }
  // The table's entry for keys at + 8 (lane % (kKeys / 8)), 0 outside the item.
  auto entry_at = [&](uint32_t at) {
    const uint32_t key8 = at + 8u * (lane % (kKeys / 8));
    return eight_of_item(key8, begin, end) ? list[key8 >> a.page_log2] : 0;
  };
  const uint32_t first = begin & ~(uint32_t)(kKeys - 1);
  uint32_t buffer = 0;
  int32_t entry = 0;
  if (begin < end) {
    // (the first step's pages are among those that held_end() has looked at: five at most)
    const uint32_t key8 = first + 8u * (lane % (kKeys / 8)), nth = (key8 >> a.page_log2) - (begin >> a.page_log2);
    const int32_t page = __shfl(held, (int)(nth & 63u));
    tile.bring(0, first, eight_of_item(key8, begin, end) ? page : 0);
    tile.settle(0);
    entry = entry_at(first + kKeys);
  }
  // (the queries have come, behind the first step's loads: a wait for them inside the loop would wait for the step's as well)
#pragma unroll
  for (int s = 0; s < D / 16; ++s) asm volatile("" : "+v"(q[s]));
  for (uint32_t base = first; begin < end && base < end; base += kKeys) {
    // This step's keys and values, and the next one's entries, have come; everybody is done with the other buffer.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const bool more = base + kKeys < end;
    if (more) {
      tile.bring(buffer ^ 1u, base + kKeys, entry);
      entry = entry_at(base + 2 * kKeys);
    }
    // Keys of a step that not every row of the block sees.  Values of keys that no row sees become zeros in shared memory,
    // whatever their place holds; where one that some rows see is not finite, the second product is taken row by row.
    const bool plain = base >= begin && base + kKeys <= block_lowest && base + kKeys <= end;
    bool by_row = false;
    if (!plain) {
      bool odd = false;
#pragma unroll 1
      for (uint32_t e = threadIdx.x; e < D * (kKeys / 8); e += 256u) {
        const uint32_t row = e / (kKeys / 8), piece = e % (kKeys / 8) ^ Tile::fv(row), k0 = base + piece * 8u;
        X8* at = reinterpret_cast<X8*>(lds + buffer * Tile::kBuffer + Tile::kKeyBytes + e * 16u);
        X8 v = *at;
        bool changed = false;
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (k0 + k < begin || k0 + k >= end) { v[k] = (T)0.0f; changed = true; }
        if (changed) *at = v;
        odd = odd || !finite16(v);
      }
      by_row = __syncthreads_or(odd);
    }
    if (base < highest) {  // (none of the wave's rows sees anything from its highest limit on)
      f32x16 x[kBlocks];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[b][e] = 0.0f;
#pragma unroll
      for (int s = 0; s < D / 16; ++s)
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) x[b] = mfma_32x32x16(tile.key(buffer, b, s), q[s], x[b]);
      feed<kBlocks * (D / 16)>();
      if (!plain) {
        const uint32_t lim = limit < end ? limit : end;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint32_t at = b * 32 + (e >> 3) * 16 + half * 8u + (e & 7), k = base + at;
            if (k < begin || k >= lim) x[b][e] = -INFINITY;
          }
      }
      float top = x[0][0];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, x[b][e]);
      top *= scale;
      // The maximum follows only where it has grown by more than 8 (weights up to 256 are as exact as up to 1); else the
      // sums need not be scaled, and the lanes of a row need not hear of each other.
      if (__any(top > m + 8.0f)) {
        top = fmaxf(top, __shfl_xor(top, 32));
        const float now = fmaxf(m, top), turn = __builtin_amdgcn_exp2f(m - (now == -INFINITY ? 0.0f : now));
        m = now;
        l *= turn;
#pragma unroll
        for (int d = 0; d < D / 32; ++d) o[d] = o[d] * turn;
      }
      const float zero = m == -INFINITY ? 0.0f : m;
      X8 p[kSteps];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          x[b][e] = __builtin_amdgcn_exp2f(fmaf(x[b][e], scale, -zero));
          sum += x[b][e];
        }
        l += sum;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          float y[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) y[k] = x[b][t * 8 + k];
          p[b * 2 + t] = narrow8<T>(y);
        }
      }
      if (!by_row) {
#pragma unroll
        for (int t = 0; t < kSteps; ++t)
#pragma unroll
          for (int d = 0; d < D / 32; ++d) o[d] = mfma_32x32x16(tile.value(buffer, d, t), p[t], o[d]);
        feed<kSteps * (D / 32)>();
      } else {
        // (rare: written to need few registers)
#pragma unroll 1
        for (uint32_t turn = 0; turn < 32u * kSteps; ++turn) {
          const uint32_t one = turn / kSteps, t = turn % kSteps, sees = __shfl(limit, (int)one);
          X8 w = p[0];
#pragma unroll
          for (uint32_t k = 1; k < (uint32_t)kSteps; ++k)
            if (t == k) w = p[k];
#pragma unroll
          for (int d = 0; d < D / 32; ++d) {
            X8 v = tile.value(buffer, d, t);
#pragma unroll
            for (int k = 0; k < 8; ++k)
              if (base + t * 16u + half * 8u + k >= sees) v[k] = (T)0.0f;
            const f32x16 y = mfma_32x32x16(v, w, o[d]);
            if (col == one) o[d] = y;
            asm volatile("" ::: "memory");
          }
        }
      }
    }
    if (more) tile.settle(buffer ^ 1u);
    buffer ^= 1u;
  }
  l += __shfl_xor(l, 32);
  if (!real) return;
  if (keys.alone) {
    const float vs = sizeof(C) == 1 && a.v_scale ? a.v_scale[head] : 1.0f;
    const float by = l == 0.0f ? 0.0f : vs / l;
    T* to = static_cast<T*>(a.out) + (uint64_t)tok * a.out_stride + (uint64_t)h * D;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t at = d * 32 + j * 8 + half * 4u;
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = l == 0.0f ? 0.0f : o[d][4 * j + i] * by;
        const auto lo = narrow2<T>(y[0], y[1]), hi = narrow2<T>(y[2], y[3]);
        typename Vec<T>::x2* w = reinterpret_cast<typename Vec<T>::x2*>(to + at);
        w[0] = lo;
        w[1] = hi;
      }
    if (a.lse && half == 0u) a.lse[(uint64_t)tok * a.n_heads + h] = l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2;
  } else {
    const uint64_t slot = (uint64_t)(is_shared ? part : a.shared_parts + part) * a.n_tok * a.n_heads + (uint64_t)tok * a.n_heads + h;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<f32x4*>(a.part_o + slot * D + d * 32 + j * 8 + half * 4u) = (f32x4){o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]};
    if (half == 0u) { a.part_ml[slot * 2] = m; a.part_ml[slot * 2 + 1] = l; }
  }
}

// Tiles, and behind them in the same launch what there is of few rows: its blocks come in as the tiles run out, and are bound
// by the pages' bytes where those are by the matrix units and shared memory.  Against a launch of their own: 160 sequences
// behind 6144 shared tokens 104 to 101 us, 20 behind five beginnings of 3372 tokens 41 to 32 us, three prompts of up to 990
// tokens (heads of 256) 32 to 23 us.  By turns with the tiles from the start, eight and eight, the first takes 119 us.
template <typename T, typename C, int D, int kKeys>
__global__ void __launch_bounds__(256, D == 256 ? 1 : 2) attention_tile_kernel(AttentionArgs a) {
  constexpr uint32_t kTile = 2 * RowTile<T, C, D, kKeys>::kBuffer, kMeet = sizeof(StreamJoin<T, D>);
  __shared__ __align__(128) char lds[kTile > kMeet ? kTile : kMeet];
  __shared__ uint32_t lowest_of[4];
  if (blockIdx.x < a.tile_blocks) tile_block<T, C, D, kKeys>(a, blockIdx.x, lds, lowest_of);
  else if (a.alone) stream_block<T, C, D, 1>(a, blockIdx.x - a.tile_blocks, nullptr);
  else stream_block<T, C, D, 4>(a, blockIdx.x - a.tile_blocks, reinterpret_cast<StreamJoin<T, D>*>(lds));
}

// Joins rows' parts.  A block takes kTokens tokens and some heads; 256 / D heads share a wave, a lane has four neighbouring
// elements of one.  With many rows each wave has heads of its own, with few (kSplit 4) the four waves share the parts of the
// same heads.  Four parts are in flight.  Bound by memory: 4 D + 8 bytes a part in, 2 D a row out.
template <typename T, typename C, int D, int kSplit, int kTokens>
__global__ void __launch_bounds__(256) attention_join_kernel(AttentionArgs a) {
  constexpr uint32_t kHeads = 256 / D, kLanes = D / 4;
  __shared__ f32x4 sum_of[kSplit][64];
  __shared__ float ml_of[kSplit][64][2];
  const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t h = (kSplit == 4 ? blockIdx.y : blockIdx.y * 4u + wave) * kHeads + lane / kLanes, at = lane % kLanes * 4u;
  const uint64_t rows = (uint64_t)a.n_tok * a.n_heads;
  uint32_t known = 0;  // the token behind the last one that `s` and `parts` are of
  SequenceSpan s{0u, 0u, 0u, 0u, 0};
  RowParts of{0u, 0u, 0u};
  for (uint32_t tok = blockIdx.x * kTokens; tok < blockIdx.x * kTokens + kTokens && tok < a.n_tok; ++tok) {
    if (tok >= known) {
      uint32_t i;
      GroupLanes groups{-1, -1, 0};
      if (a.n_groups) groups = groups_from(a, 0u);
      s = sequence_of(a, tok, i);
      const bool mine = tok >= s.tok0 && tok - s.tok0 < s.n_q;
      of = mine ? row_parts(a, s.len, shared_of(a, i, groups)) : RowParts{0u, 1u, 0u};  // (of no sequence: left alone)
      known = mine ? s.tok0 + s.n_q : tok + 1u;
    }
    if (of.n_shared == 0u && of.n_own == 1u) {  // (written already)
      if (known > tok + 1u) tok = known - 1u;
      continue;
    }
    const bool real = h < a.n_heads;
    const uint64_t row = (uint64_t)tok * a.n_heads + (real ? h : 0u);
    const uint32_t parts = of.n_shared + of.n_own;
    float m = -INFINITY, l = 0.0f;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t p0 = kSplit == 4 ? wave : 0u; p0 < parts; p0 += 4u * kSplit) {
      f32x4 v[4];
      float pm[4], pl[4];
#pragma unroll
      for (uint32_t k = 0; k < 4u; ++k) {
        const uint32_t p = p0 + k * kSplit < parts ? p0 + k * kSplit : p0;
        const uint64_t slot = (uint64_t)(p < of.n_shared ? p : a.shared_parts + (p - of.n_shared)) * rows + row;
        const f32x2 ml = *reinterpret_cast<const f32x2*>(a.part_ml + slot * 2);
        v[k] = *reinterpret_cast<const f32x4*>(a.part_o + slot * D + at);
        pm[k] = p0 + k * kSplit < parts ? ml[0] : -INFINITY;
        pl[k] = ml[1];
      }
      const float top = fmaxf(fmaxf(fmaxf(m, pm[0]), fmaxf(pm[1], pm[2])), pm[3]), zero = top == -INFINITY ? 0.0f : top;
      const float turn = __builtin_amdgcn_exp2f(m - zero);
      m = top;
      l *= turn;
      acc = acc * turn;
#pragma unroll
      for (uint32_t k = 0; k < 4u; ++k) {
        const float w = __builtin_amdgcn_exp2f(pm[k] - zero);
        if (p0 + k * kSplit >= parts) break;
        l = fmaf(pl[k], w, l);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = fmaf(v[k][e], w, acc[e]);
      }
    }
    if constexpr (kSplit == 4) {
      __syncthreads();
      sum_of[wave][lane] = acc;
      ml_of[wave][lane][0] = m;
      ml_of[wave][lane][1] = l;
      __syncthreads();
      if (wave != 0u) continue;
      m = fmaxf(fmaxf(ml_of[0][lane][0], ml_of[1][lane][0]), fmaxf(ml_of[2][lane][0], ml_of[3][lane][0]));
      const float zero = m == -INFINITY ? 0.0f : m;
      l = 0.0f;
      acc = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float turn = __builtin_amdgcn_exp2f(ml_of[w][lane][0] - zero);
        l = fmaf(ml_of[w][lane][1], turn, l);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = fmaf(sum_of[w][lane][e], turn, acc[e]);
      }
    }
    if (!real) continue;
    const float vs = sizeof(C) == 1 && a.v_scale ? a.v_scale[h / a.group] : 1.0f;
    const float by = l == 0.0f ? 0.0f : vs / l;
    typename Vec<T>::x2* to = reinterpret_cast<typename Vec<T>::x2*>(static_cast<T*>(a.out) + (uint64_t)tok * a.out_stride + (uint64_t)h * D + at);
    to[0] = l == 0.0f ? narrow2<T>(0.0f, 0.0f) : narrow2<T>(acc[0] * by, acc[1] * by);
    to[1] = l == 0.0f ? narrow2<T>(0.0f, 0.0f) : narrow2<T>(acc[2] * by, acc[3] * by);
    if (a.lse && at == 0u) a.lse[row] = l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2;
  }
}

}  // namespace maaso
