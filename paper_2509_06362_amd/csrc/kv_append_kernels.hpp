// New tokens' queries, keys and values: norm of each head, position rotation, and the write into the cache's
// pages, in one pass over the data.  Bound by memory (2 bytes in and 2 out per element, some 7 operations): 7000 tokens of 32
// and 8 heads of 128 in 23 us, 4.7 TB/s, of which a copy reaches 4.8 (29 us before queries of more than the L2s hold, 32 MiB,
// were written past them); 64 tokens in 5 us, a launch's time.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/maaso_instance.h"
#include "element_types.hpp"
#include "kv_pages_kernels.hpp"

namespace maaso {

struct AppendArgs {
  const void* q;
  const void* k;
  const void* v;
  void* q_out;
  const void* q_weight;
  const void* k_weight;
  const float* cos_sin;
  const int32_t* pos;
  const int64_t* slot;
  const float* k_scale;
  const float* v_scale;
  char* k_pages;  // the layer's
  char* v_pages;
  uint64_t q_stride, k_stride, v_stride, q_out_stride, page_stride;  // elements
  uint64_t n_slots;
  uint32_t n_tok, n_heads, n_kv_heads, rotary, n_pos, page_log2;
  uint32_t value_blocks;  // blocks that take values, the longer work, before those that take heads; 0: with the heads
  float eps;
  bool past;  // queries are written past the caches
  uint32_t* status;
};

// Eight elements from p on, whatever its alignment: one 16-byte access all the same, and as fast where p is a multiple of 16.
template <typename T> struct Eight {
  typedef typename Vec<T>::x8 x8;
  struct __attribute__((packed, aligned(2))) at { x8 v; };
};
template <typename T> __device__ inline typename Vec<T>::x8 load8(const T* p) { return reinterpret_cast<const typename Eight<T>::at*>(p)->v; }
template <typename T> __device__ inline void store8(T* p, typename Vec<T>::x8 v, bool past) {
  typedef uint32_t sixteen __attribute__((ext_vector_type(4), aligned(2)));
  if (past) {
    keep_apart();
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<sixteen*>(p));
    keep_apart();
  } else {
    reinterpret_cast<typename Eight<T>::at*>(p)->v = v;
  }
}

// One element of a page, in the cache's type; scale: what 8 bits are multiplied by.
template <typename T, typename C>
__device__ inline void store_one(C* p, T x, float scale) {
  if constexpr (sizeof(C) == 1) p->bits = (uint8_t)e4m3_pack4((float)x / scale, 0.0f, 0.0f, 0.0f);
  else *p = x;
}

// Eight lanes per 64 elements of a head, eight elements a lane: a head's sum of squares is a few lane exchanges, and the
// rotation's partner of an element lies at the same place of another lane (or in the lane, interleaved).  Values, where
// kValues, are taken the same way and written element by element: their places in a page lie page_size apart.  A lane has
// pieces of kAppendHeads heads, all asked for before the first is worked on: with one alone too few bytes were on their way.
constexpr uint32_t kAppendHeads = 2;

template <typename T, typename C, int D, bool kInterleaved>
__device__ inline void append_heads(const AppendArgs& a, uint32_t block, bool values) {
  constexpr uint32_t kLanes = D / 8, kPer = 256 / kLanes;
  const uint32_t lane = threadIdx.x % kLanes, heads = a.n_heads + a.n_kv_heads * (values ? 2u : 1u);
  const uint64_t first = (uint64_t)block * (kPer * kAppendHeads);
  const uint32_t t0 = first >> 32 ? (uint32_t)(first / heads) : (uint32_t)first / heads, r0 = (uint32_t)(first - (uint64_t)t0 * heads);
  typename Vec<T>::x8 raw[kAppendHeads];
  uint32_t toks[kAppendHeads], hs[kAppendHeads];
  bool inside[kAppendHeads];
#pragma unroll
  for (uint32_t u = 0; u < kAppendHeads; ++u) {
    const uint32_t r = r0 + u * kPer + threadIdx.x / kLanes, t = t0 + r / heads, h = r % heads;
    inside[u] = t < a.n_tok;
    const uint32_t tok = inside[u] ? t : a.n_tok - 1u;  // (lanes past the end take part in the exchanges)
    toks[u] = tok;
    hs[u] = h;
    const uint32_t hk = h < a.n_heads ? 0u : h - a.n_heads;
    const T* src = h < a.n_heads ? static_cast<const T*>(a.q) + tok * a.q_stride + (uint64_t)h * D
                   : hk >= a.n_kv_heads ? static_cast<const T*>(a.v) + tok * a.v_stride + (uint64_t)(hk - a.n_kv_heads) * D
                                        : static_cast<const T*>(a.k) + tok * a.k_stride + (uint64_t)hk * D;
    raw[u] = load8<T>(src + lane * 8u);
  }
#pragma unroll
  for (uint32_t u = 0; u < kAppendHeads; ++u) {
    const uint32_t tok = toks[u], h = hs[u];
    const bool is_q = h < a.n_heads, is_v = h >= a.n_heads + a.n_kv_heads;
    const uint32_t hk = is_q ? 0u : is_v ? h - a.n_heads - a.n_kv_heads : h - a.n_heads;
    float x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = (float)raw[u][k];
    const T* weight = static_cast<const T*>(is_q ? a.q_weight : a.k_weight);
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum = fmaf(x[k], x[k], sum);
#pragma unroll
    for (uint32_t d = 1; d < kLanes; d <<= 1) sum += __shfl_xor(sum, d);
    if (weight && !is_v) {
      const float by = rsqrtf(sum * (1.0f / D) + a.eps);
      const auto w = load8<T>(weight + lane * 8u);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = x[k] * by * (float)w[k];
    }
    if (a.rotary != 0u) {
      int32_t pos = a.pos[tok];
      if (pos < 0 || (uint32_t)pos >= a.n_pos) {
        if (lane == 0) raise(a.status, MAASO_INST_BAD_POS);
        pos = pos < 0 ? 0 : (int32_t)a.n_pos - 1;
      }
      const float* cs = a.cos_sin + (uint64_t)pos * a.rotary;
      const uint32_t half = a.rotary / 2u;
      const bool turns = lane * 8u < a.rotary && !is_v;
      if constexpr (kInterleaved) {
        if (turns) {
          const f32x4 c = *reinterpret_cast<const f32x4*>(cs + lane * 4u), s = *reinterpret_cast<const f32x4*>(cs + half + lane * 4u);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float v = x[2 * k], w = x[2 * k + 1];
            x[2 * k] = v * c[k] - w * s[k];
            x[2 * k + 1] = w * c[k] + v * s[k];
          }
        }
      } else {
        const uint32_t step = half / 8u;
        const bool second = lane >= step;
        const uint32_t other = turns ? (second ? lane - step : lane + step) : lane;
        float y[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = __shfl(x[k], (int)other, (int)kLanes);
        if (turns) {
          const uint32_t at = (second ? lane - step : lane) * 8u;
          const f32x4 c0 = *reinterpret_cast<const f32x4*>(cs + at), c1 = *reinterpret_cast<const f32x4*>(cs + at + 4u);
          const f32x4 s0 = *reinterpret_cast<const f32x4*>(cs + half + at), s1 = *reinterpret_cast<const f32x4*>(cs + half + at + 4u);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float c = k < 4 ? c0[k & 3] : c1[k & 3], s = k < 4 ? s0[k & 3] : s1[k & 3];
            x[k] = second ? x[k] * c + y[k] * s : x[k] * c - y[k] * s;
          }
        }
      }
    }
    if (!inside[u]) continue;
    if (is_q) {
      store8<T>(static_cast<T*>(a.q_out) + tok * a.q_out_stride + (uint64_t)h * D + lane * 8u, narrow8<T>(x), a.past);
      continue;
    }
    const int64_t slot = a.slot[tok];
    if (slot < 0) continue;
    if ((uint64_t)slot >= a.n_slots) {
      if (lane == 0) raise(a.status, MAASO_INST_BAD_PAGE);
      continue;
    }
    const uint64_t page = (uint64_t)slot >> a.page_log2;
    const uint32_t place = (uint32_t)slot & ((1u << a.page_log2) - 1u);
    if (is_v) {
      C* to = reinterpret_cast<C*>(a.v_pages) + page * a.page_stride + (((uint64_t)hk * D + lane * 8u) << a.page_log2) + place;
      const float scale = sizeof(C) == 1 && a.v_scale ? a.v_scale[hk] : 1.0f;
#pragma unroll
      for (int k = 0; k < 8; ++k) store_one<T, C>(to + ((uint64_t)k << a.page_log2), raw[u][k], scale);
      continue;
    }
    C* to = reinterpret_cast<C*>(a.k_pages) + page * a.page_stride + (((uint64_t)hk << a.page_log2) + place) * D + lane * 8u;
    if constexpr (sizeof(C) == 1) {
      const float s = a.k_scale ? a.k_scale[hk] : 1.0f;
      u32x2 b;
      b[0] = e4m3_pack4(x[0] / s, x[1] / s, x[2] / s, x[3] / s);
      b[1] = e4m3_pack4(x[4] / s, x[5] / s, x[6] / s, x[7] / s);
      *reinterpret_cast<u32x2*>(to) = b;
    } else {
      *reinterpret_cast<typename Vec<T>::x8*>(to) = narrow8<T>(x);
    }
  }
}

// Values of many tokens: a block turns 64 tokens by 64 elements of a head through shared memory.  Up to eight tokens
// that follow each other within eight places of a page are one store of eight elements, others go one by one.
constexpr uint32_t kTurnTokens = 64, kTurnPad = 66;

template <typename T, typename C, int D>
__device__ inline void append_values(const AppendArgs& a, uint32_t block) {
  __shared__ T tile[kTurnTokens * kTurnPad];
  const uint32_t per_token = a.n_kv_heads * (D / 64);
  const uint32_t t0 = block / per_token * kTurnTokens, hd = block % per_token;
  const uint32_t hk = hd / (D / 64), d0 = hd % (D / 64) * 64u;
  const uint32_t n = a.n_tok - t0 < kTurnTokens ? a.n_tok - t0 : kTurnTokens;
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
  const uint32_t t = threadIdx.x / 8u, d = threadIdx.x % 8u * 8u, t2 = t + 32u < n ? t + 32u : n - 1u;  // (past the end: the last again)
  const T* src = static_cast<const T*>(a.v) + (uint64_t)hk * D + d0 + d;
  const auto x = load8<T>(src + (t0 + (t < n ? t : n - 1u)) * a.v_stride), y = load8<T>(src + (t0 + t2) * a.v_stride);
  int64_t slot = lane < n ? a.slot[t0 + lane] : -1;
#pragma unroll
  for (int k = 0; k < 8; ++k) tile[t * kTurnPad + d + k] = x[k];
#pragma unroll
  for (int k = 0; k < 8; ++k) tile[(t + 32u) * kTurnPad + d + k] = y[k];
  if (slot >= 0 && (uint64_t)slot >= a.n_slots) {
    if (wave == 0) raise(a.status, MAASO_INST_BAD_PAGE);
    slot = -1;
  }
  const int64_t before = __shfl_up(slot, 1);
  const uint64_t starts = __ballot(lane == 0 || slot < 0 || (slot & 7) == 0 || slot != before + 1);
  __syncthreads();
  const float scale = sizeof(C) == 1 && a.v_scale ? a.v_scale[hk] : 1.0f;
  uint32_t job = 0;
  for (uint64_t left = starts; left; ++job) {
    const uint32_t begin = (uint32_t)__builtin_ctzll(left);
    left &= left - 1u;
    const uint32_t end = left ? (uint32_t)__builtin_ctzll(left) : 64u;
    if ((job & 3u) != wave) continue;
    const int64_t s = __shfl(slot, (int)begin);
    if (s < 0) continue;
    C* to = reinterpret_cast<C*>(a.v_pages) + (uint64_t)(s >> a.page_log2) * a.page_stride +
            (((uint64_t)hk * D + d0 + lane) << a.page_log2) + (uint32_t)(s & ((1 << a.page_log2) - 1));
    if (end - begin == 8u) {
      typename Vec<T>::x8 x;
#pragma unroll
      for (uint32_t k = 0; k < 8u; ++k) x[k] = tile[(begin + k) * kTurnPad + lane];
      if constexpr (sizeof(C) == 1) {
        u32x2 b;
        b[0] = e4m3_pack4((float)x[0] / scale, (float)x[1] / scale, (float)x[2] / scale, (float)x[3] / scale);
        b[1] = e4m3_pack4((float)x[4] / scale, (float)x[5] / scale, (float)x[6] / scale, (float)x[7] / scale);
        *reinterpret_cast<u32x2*>(to) = b;
      } else {
        *reinterpret_cast<typename Vec<T>::x8*>(to) = x;
      }
    } else {
      for (uint32_t k = 0; begin + k < end; ++k) store_one<T, C>(to + k, tile[(begin + k) * kTurnPad + lane], scale);
    }
  }
}

template <typename T, typename C, int D, bool kInterleaved>
__global__ void __launch_bounds__(256) append_kernel(AppendArgs a) {
  if (blockIdx.x < a.value_blocks) append_values<T, C, D>(a, blockIdx.x);
  else append_heads<T, C, D, kInterleaved>(a, blockIdx.x - a.value_blocks, a.value_blocks == 0u);
}

}  // namespace maaso
