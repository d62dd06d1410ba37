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
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/maaso_instance.h"
#include "element_types.hpp"
#include "kv_pages_kernels.hpp"

namespace maaso {

constexpr float kLn2 = 0.693147180559945309f;
constexpr uint32_t kStreamRows = 16;  // rows of an item
constexpr uint32_t kStreamKeys = 32;  // keys of a wave's step

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
  uint32_t max_q, max_len, max_shared;
  uint32_t own_chunk, shared_chunk;    // keys of a part, multiples of kStreamKeys
  uint32_t own_parts, shared_parts;    // most parts of a row
  uint32_t own_tiles, shared_tiles;    // most tiles of rows
  uint32_t shared_blocks;              // blocks that take shared parts; those behind them take own ones
  float scale_log2;
  // workspace, where a row has several parts
  float* part_o;   // [part][n_tok * n_heads][D]
  float* part_ml;  // [part][n_tok * n_heads][2]
  uint32_t* status;
};

// What a sequence or a group has of rows and keys, from the device's arrays; everything within its bounds.
struct SequenceSpan {
  uint32_t row, tok0, n_q, len;
};

__device__ inline SequenceSpan sequence_span(const AttentionArgs& a, uint32_t i) {
  SequenceSpan s{0u, 0u, 0u, 0u};
  const int32_t q0 = a.q_start[i], q1 = a.q_start[i + 1];
  if (q0 < 0 || q1 < q0 || (uint32_t)q1 > a.n_tok) { raise(a.status, MAASO_INST_BAD_BOUND); return s; }
  const int32_t row = a.rows ? a.rows[i] : (int32_t)i;
  s.tok0 = (uint32_t)q0;
  s.n_q = (uint32_t)(q1 - q0);
  if (s.n_q > a.max_q) { raise(a.status, MAASO_INST_BAD_BOUND); s.n_q = a.max_q; }
  if (row < 0 || (uint32_t)row >= a.n_rows) { raise(a.status, MAASO_INST_BAD_ROW); return s; }
  s.row = (uint32_t)row;
  const int32_t len = a.length[row];
  if (len < 0 || (uint64_t)len > (uint64_t)a.width << a.page_log2) { raise(a.status, MAASO_INST_BAD_ROW); return s; }
  s.len = (uint32_t)len;
  if (s.len > a.max_len) { raise(a.status, MAASO_INST_BAD_BOUND); s.len = a.max_len; }
  return s;
}

// Keys that query j of the span sees.
__device__ inline uint32_t seen_keys(const SequenceSpan& s, uint32_t q_all, uint32_t j) {
  const int64_t limit = (int64_t)s.len - q_all + j + 1;
  return limit < 0 ? 0u : (uint32_t)limit;
}

// Keys of group g's common part: what the caller says, within the bound and the first sequence's row.
__device__ inline uint32_t group_keys(const AttentionArgs& a, uint32_t g) {
  const int32_t v = a.shared[g], f = a.group_start[g];
  if (v <= 0 || f < 0 || (uint32_t)f >= a.n) return 0u;
  const int32_t row = a.rows ? a.rows[f] : f;
  if (row < 0 || (uint32_t)row >= a.n_rows) return 0u;
  const int32_t len = a.length[row];
  if (len < 0 || (uint64_t)len > (uint64_t)a.width << a.page_log2) return 0u;
  const uint32_t most = a.max_shared < a.max_len ? a.max_shared : a.max_len;
  uint32_t keys = (uint32_t)v < (uint32_t)len ? (uint32_t)v : (uint32_t)len;
  if (keys < (uint32_t)v || keys > most) raise(a.status, MAASO_INST_BAD_BOUND);
  return keys < most ? keys : most;
}

// Tokens that sequence i begins with like its group, 0 outside every group.
__device__ inline uint32_t shared_of(const AttentionArgs& a, uint32_t i) {
  if (a.n_groups == 0u || a.max_shared == 0u) return 0u;
  uint32_t lo = 0, hi = a.n_groups;
  while (hi - lo > 1u) {
    const uint32_t mid = (lo + hi) >> 1;
    if (a.group_start[mid] <= (int32_t)i) lo = mid; else hi = mid;
  }
  const int32_t f = a.group_start[lo], e = a.group_start[lo + 1];
  if (f < 0 || f > (int32_t)i || e <= (int32_t)i || (uint32_t)e > a.n) return 0u;
  return group_keys(a, lo);
}

// The sequence of token t: the last one that begins at t or before.
__device__ inline uint32_t sequence_of(const AttentionArgs& a, uint32_t t) {
  if (a.max_q == 1u && a.n_tok == a.n) return t;
  uint32_t lo = 0, hi = a.n;
  while (hi - lo > 1u) {
    const uint32_t mid = (lo + hi) >> 1;
    if ((uint32_t)a.q_start[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}

// Item `tile` counted through all sequences' (or groups') tiles of `rows` rows: which one, and its first row there.
// Taken by every lane of a wave alike.
__device__ inline bool find_tile(const AttentionArgs& a, bool groups, uint32_t rows, uint32_t tile, uint32_t& which, uint32_t& row0) {
  const uint32_t count = groups ? a.n_groups : a.n, lane = threadIdx.x & 63u;
  uint32_t before = 0;
  for (uint32_t base = 0; base < count; base += 64u) {
    const uint32_t i = base + lane;
    uint32_t tiles = 0;
    if (i < count) {
      uint32_t f = i, e = i + 1u;
      bool good = true;
      if (groups) {
        const int32_t gf = a.group_start[i], ge = a.group_start[i + 1];
        good = gf >= 0 && ge >= gf && (uint32_t)ge <= a.n;
        f = good ? (uint32_t)gf : 0u;
        e = good ? (uint32_t)ge : 0u;
      }
      const int32_t q0 = a.q_start[f], q1 = a.q_start[e];
      good = good && q0 >= 0 && q1 >= q0 && (uint32_t)q1 <= a.n_tok;
      if (!good) raise(a.status, MAASO_INST_BAD_BOUND);
      else tiles = (uint32_t)(((uint64_t)(uint32_t)(q1 - q0) * a.group + rows - 1u) / rows);
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

template <typename T, typename C> struct KeyLoad;
template <typename T> struct KeyLoad<T, T> {
  using raw = typename Vec<T>::x8;
  static __device__ inline typename Vec<T>::x8 wide(raw r) { return r; }
};
template <typename T> struct KeyLoad<T, E4m3> {
  using raw = u32x2;
  static __device__ inline typename Vec<T>::x8 wide(raw r) { return widen8<T>(r); }
};

template <typename V> __device__ inline bool finite16(V v) {
  bool f = true;
#pragma unroll
  for (int k = 0; k < 8; ++k) f = f && __builtin_isfinite((float)v[k]);
  return f;
}

// Keys [begin, end) of page list `list` against one tile of rows, by this wave's steps begin + (step0 + i * stride) * 32.
template <typename T, typename C, int D>
struct StreamTile {
  using X8 = typename Vec<T>::x8;
  X8 q[D / 32];
  f32x4 o[D / 16];
  float m, l;

  __device__ inline void clear() {
#pragma unroll
    for (int d = 0; d < D / 16; ++d) o[d] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    m = -INFINITY;
    l = 0.0f;
  }

  // limit: keys that this lane's row sees; lowest, highest: over all rows of the tile
  __device__ inline void run(const AttentionArgs& a, const int32_t* list, uint32_t head, float scale, uint32_t begin, uint32_t end,
                             uint32_t first, uint32_t stride, uint32_t limit, uint32_t lowest) {
    using L = KeyLoad<T, C>;
    const uint32_t lane = threadIdx.x & 63u, col = lane & 15u, g = lane >> 4, per = 1u << a.page_log2;
    const C* kp = reinterpret_cast<const C*>(a.k_pages) + ((uint64_t)head << a.page_log2) * D;
    const C* vp = reinterpret_cast<const C*>(a.v_pages) + ((uint64_t)head << a.page_log2) * D;
    for (uint32_t base = (begin & ~(kStreamKeys - 1u)) + first * kStreamKeys; base < end; base += stride * kStreamKeys) {
      const uint32_t key8 = base + 8u * g;  // this lane's eight keys of the second product
      int32_t page = 0;
      bool held = false;
      if (key8 < end && key8 + 8u > begin) {
        page = list[key8 >> a.page_log2];
        held = page >= 0 && (uint32_t)page < a.n_pages;
        if (!held) { page = 0; raise(a.status, MAASO_INST_BAD_PAGE); }
      }
      const int from = (int)((col >> 2) << 4);
      const int32_t kpage = __shfl(page, from);
      const uint32_t row = (base + 8u * (col >> 2) + (col & 3u)) & (per - 1u);
      const C* kr = kp + (uint64_t)(uint32_t)kpage * a.page_stride + (uint64_t)row * D + g * 8u;
      const C* vr = vp + (uint64_t)(uint32_t)page * a.page_stride + (key8 & (per - 1u)) + ((uint64_t)col << a.page_log2);
      typename L::raw kr0[D / 32], kr1[D / 32], vv[D / 16];
#pragma unroll
      for (int s = 0; s < D / 32; ++s) {
        kr0[s] = *reinterpret_cast<const typename L::raw*>(kr + s * 32);
        kr1[s] = *reinterpret_cast<const typename L::raw*>(kr + 4 * D + s * 32);
      }
#pragma unroll
      for (int d = 0; d < D / 16; ++d) vv[d] = *reinterpret_cast<const typename L::raw*>(vr + ((uint64_t)(d * 16) << a.page_log2));
      f32x4 s0 = {0.0f, 0.0f, 0.0f, 0.0f}, s1 = s0;
#pragma unroll
      for (int s = 0; s < D / 32; ++s) {
        s0 = mfma_16x16x32(L::wide(kr0[s]), q[s], s0);
        s1 = mfma_16x16x32(L::wide(kr1[s]), q[s], s1);
      }
      float x[8];
      const bool inner = base >= begin && base + kStreamKeys <= lowest && base + kStreamKeys <= end;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[k] = s0[k] * scale;
        x[k + 4] = s1[k] * scale;
      }
      const bool plain = inner && __all(held);
      if (!plain) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t key = key8 + k;
          if (!held || key < begin || key >= end || key >= limit) x[k] = -INFINITY;
        }
      }
      float top = x[0];
#pragma unroll
      for (int k = 1; k < 8; ++k) top = fmaxf(top, x[k]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float now = fmaxf(m, top), zero = now == -INFINITY ? 0.0f : now;
      const float turn = __builtin_amdgcn_exp2f(m - zero);
      float p[8], sum = 0.0f;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        p[k] = __builtin_amdgcn_exp2f(x[k] - zero);
        sum += p[k];
      }
      l = fmaf(l, turn, sum);
      m = now;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) o[d] = o[d] * turn;
      const X8 w = narrow8<T>(p);
      X8 v[D / 16];
#pragma unroll
      for (int d = 0; d < D / 16; ++d) v[d] = L::wide(vv[d]);
      if (!plain) {
        // Keys that no row sees: zeros, whatever their place holds.
        bool odd = false;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const uint32_t key = key8 + k;
            if (!held || key < begin || key >= end) v[d][k] = (T)0.0f;
          }
          odd = odd || !finite16(v[d]);
        }
        if (__any(odd)) {
          // A value that is not finite, which some rows see and others do not: row by row.
          for (int r = 0; r < 16; ++r) {
            const uint32_t sees = __shfl(limit, r);
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
              X8 vr1 = v[d];
#pragma unroll
              for (int k = 0; k < 8; ++k)
                if (key8 + k >= sees) vr1[k] = (T)0.0f;
              const f32x4 t = mfma_16x16x32(vr1, w, o[d]);
              if (col == (uint32_t)r) o[d] = t;
            }
          }
          continue;
        }
      }
#pragma unroll
      for (int d = 0; d < D / 16; ++d) o[d] = mfma_16x16x32(v[d], w, o[d]);
    }
  }
};

template <typename T, typename C, int D>
__global__ void __launch_bounds__(256) attention_stream_kernel(AttentionArgs a) {
  using X8 = typename Vec<T>::x8;
  constexpr int kPad = D + 4;
  __shared__ float so[4][16][kPad];
  __shared__ float sm[4][16], sl[4][16];
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, col = lane & 15u, g = lane >> 4;
  // block -> (part, head, tile)
  const bool is_shared = blockIdx.x < a.shared_blocks;
  uint32_t id = is_shared ? blockIdx.x : blockIdx.x - a.shared_blocks;
  const uint32_t head = id % a.n_kv_heads;
  id /= a.n_kv_heads;
  const uint32_t tiles = is_shared ? a.shared_tiles : a.own_tiles;
  const uint32_t tile = id % tiles, part = id / tiles;
  uint32_t which, row0;
  if (!is_shared && a.max_q * a.group <= kStreamRows) { which = tile; row0 = 0; }
  else if (!find_tile(a, is_shared, kStreamRows, tile, which, row0)) return;
  // the tile's rows and keys
  uint32_t tok0, n_rows, begin, end, page_row;
  SequenceSpan span{0u, 0u, 0u, 0u};
  uint32_t q_all = 0;
  if (is_shared) {
    const uint32_t f = (uint32_t)a.group_start[which], e = (uint32_t)a.group_start[which + 1];  // (find_tile has checked them)
    tok0 = (uint32_t)a.q_start[f];
    n_rows = ((uint32_t)a.q_start[e] - tok0) * a.group;
    page_row = a.rows ? (uint32_t)a.rows[f] : f;  // (group_keys has checked it where there are keys)
    const uint32_t keys = group_keys(a, which);
    begin = part * a.shared_chunk;
    end = begin + a.shared_chunk < keys ? begin + a.shared_chunk : keys;
  } else {
    span = sequence_span(a, which);
    q_all = span.n_q;
    tok0 = span.tok0;
    n_rows = span.n_q * a.group;
    page_row = span.row;
    const uint32_t own = shared_of(a, which);
    const uint64_t b = (uint64_t)own + (uint64_t)part * a.own_chunk;
    begin = b < span.len ? (uint32_t)b : span.len;
    end = span.len - begin < a.own_chunk ? span.len : begin + a.own_chunk;
  }
  // A block without keys has nothing to join, except that rows without any part at all are written by part 0.
  const bool direct = a.part_o == nullptr;
  if (begin >= end && !(direct && part == 0)) return;
  const uint32_t r = row0 + col;
  const bool real = r < n_rows;
  const uint32_t tok = tok0 + (real ? r : row0) / a.group, h = head * a.group + (real ? r : row0) % a.group;
  if (row0 >= n_rows) return;
  uint32_t limit;
  if (is_shared) {
    const uint32_t i = sequence_of(a, tok);
    const SequenceSpan s = sequence_span(a, i);
    limit = seen_keys(s, s.n_q, tok - s.tok0);
  } else {
    limit = seen_keys(span, q_all, tok - tok0);
  }
  uint32_t lowest = limit, highest = limit;
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) {
    const uint32_t x = __shfl_xor(lowest, d), y = __shfl_xor(highest, d);
    lowest = x < lowest ? x : lowest;
    highest = y > highest ? y : highest;
  }
  if (end > highest) end = highest;
  StreamTile<T, C, D> st;
  const T* qp = static_cast<const T*>(a.q) + (uint64_t)tok * a.q_stride + (uint64_t)h * D + g * 8u;
#pragma unroll
  for (int s = 0; s < D / 32; ++s) st.q[s] = *reinterpret_cast<const X8*>(qp + s * 32);
  st.clear();
  const float scale = a.scale_log2 * (sizeof(C) == 1 && a.k_scale ? a.k_scale[head] : 1.0f);
  if (begin < end)
    st.run(a, a.table + (uint64_t)page_row * a.width, head, scale, begin, end, wave, 4u, limit, lowest);
  // join the waves
  float l = st.l;
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
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
  if (row0 + orow >= n_rows) return;
  float mm = -INFINITY, ll = 0.0f;
#pragma unroll
  for (int w = 0; w < 4; ++w) mm = fmaxf(mm, sm[w][orow]);
  const float zero = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
  for (int w = 0; w < 4; ++w) ll += sl[w][orow] * __builtin_amdgcn_exp2f(sm[w][orow] - zero);
  float acc[D / 16];
#pragma unroll
  for (int k = 0; k < D / 16; ++k) acc[k] = (so[0][orow][at + k] + so[1][orow][at + k]) + (so[2][orow][at + k] + so[3][orow][at + k]);
  const uint32_t otok = tok0 + (row0 + orow) / a.group, oh = head * a.group + (row0 + orow) % a.group;
  if (direct) {
    const float vs = sizeof(C) == 1 && a.v_scale ? a.v_scale[head] : 1.0f;
    const float by = ll == 0.0f ? 0.0f : vs / ll;
    T* to = static_cast<T*>(a.out) + (uint64_t)otok * a.out_stride + (uint64_t)oh * D + at;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) to[k] = (T)(ll == 0.0f ? 0.0f : acc[k] * by);
    if (a.lse && at == 0) a.lse[(uint64_t)otok * a.n_heads + oh] = ll == 0.0f ? -INFINITY : (mm + log2f(ll)) * kLn2;
  } else {
    const uint64_t slot = (uint64_t)(is_shared ? part : a.shared_parts + part) * a.n_tok * a.n_heads + (uint64_t)otok * a.n_heads + oh;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) a.part_o[slot * D + at + k] = acc[k];
    if (at == 0) { a.part_ml[slot * 2] = mm; a.part_ml[slot * 2 + 1] = ll; }
  }
}

// Joins a row's parts: a wave for each (token, head).
template <typename T, typename C, int D>
__global__ void __launch_bounds__(256) attention_join_kernel(AttentionArgs a) {
  const uint32_t lane = threadIdx.x & 63u;
  const uint64_t row = (uint64_t)blockIdx.x * 4u + (threadIdx.x >> 6), rows = (uint64_t)a.n_tok * a.n_heads;
  if (row >= rows) return;
  const uint32_t tok = (uint32_t)(row / a.n_heads), h = (uint32_t)(row % a.n_heads);
  const uint32_t i = sequence_of(a, tok);
  const SequenceSpan s = sequence_span(a, i);
  const uint32_t own0 = shared_of(a, i), j = tok - s.tok0;
  const bool mine = tok >= s.tok0 && j < s.n_q;
  // parts that were written: those of the group's keys, those of the sequence's
  uint32_t n_shared = 0, n_own = 0;
  if (mine && own0) n_shared = (own0 + a.shared_chunk - 1u) / a.shared_chunk;
  if (mine && s.len > own0) n_own = (s.len - own0 + a.own_chunk - 1u) / a.own_chunk;
  float m = -INFINITY;
  const uint32_t parts = n_shared + n_own;
  auto slot = [&](uint32_t p) { return (uint64_t)(p < n_shared ? p : a.shared_parts + (p - n_shared)) * rows + row; };
  for (uint32_t p = lane; p < parts; p += 64u) m = fmaxf(m, a.part_ml[slot(p) * 2]);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  const float zero = m == -INFINITY ? 0.0f : m;
  float l = 0.0f, acc[D / 64];
#pragma unroll
  for (int k = 0; k < D / 64; ++k) acc[k] = 0.0f;
  for (uint32_t p = 0; p < parts; ++p) {
    const uint64_t at = slot(p);
    const float turn = __builtin_amdgcn_exp2f(a.part_ml[at * 2] - zero);
    l = fmaf(a.part_ml[at * 2 + 1], turn, l);
#pragma unroll
    for (int k = 0; k < D / 64; ++k) acc[k] = fmaf(a.part_o[at * D + lane * (D / 64) + k], turn, acc[k]);
  }
  const float vs = sizeof(C) == 1 && a.v_scale ? a.v_scale[h / a.group] : 1.0f;
  const float by = l == 0.0f ? 0.0f : vs / l;
  T* to = static_cast<T*>(a.out) + (uint64_t)tok * a.out_stride + (uint64_t)h * D + lane * (D / 64);
#pragma unroll
  for (int k = 0; k < D / 64; ++k) to[k] = (T)(l == 0.0f ? 0.0f : acc[k] * by);
  if (a.lse && lane == 0) a.lse[row] = l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2;
}

}  // namespace maaso
