// New tokens' queries, keys and values: norm of each head, position rotation, and the write into the cache's
// pages, in one pass over the data.  Bound by memory (2 bytes in and 2 out per element, some 7 operations).
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
  uint32_t head_blocks;  // blocks that take heads; those behind them take values
  float eps;
  uint32_t* status;
};

// Eight elements from p on, which is a multiple of 16 bytes where kWide.
template <typename T, bool kWide>
__device__ inline typename Vec<T>::x8 load8(const T* p) {
  if constexpr (kWide) return *reinterpret_cast<const typename Vec<T>::x8*>(p);
  typename Vec<T>::x8 r;
#pragma unroll
  for (int k = 0; k < 8; ++k) r[k] = p[k];
  return r;
}

template <typename T, bool kWide>
__device__ inline void store8(T* p, typename Vec<T>::x8 v) {
  if constexpr (kWide) { *reinterpret_cast<typename Vec<T>::x8*>(p) = v; return; }
#pragma unroll
  for (int k = 0; k < 8; ++k) p[k] = v[k];
}

// One element of a page, in the cache's type.
template <typename T, typename C>
__device__ inline void store_one(C* p, T x, float inv) {
  if constexpr (sizeof(C) == 1) p->bits = (uint8_t)e4m3_pack4((float)x / inv, 0.0f, 0.0f, 0.0f);
  else *p = x;
}

// Eight lanes per 64 elements of a head, eight elements a lane: a head's sum of squares is a few lane exchanges, and the
// rotation's partner of an element lies at the same place of another lane (or in the lane, interleaved).  Values, where
// kValues, are taken the same way and written element by element: their places in a page lie page_size apart.
template <typename T, typename C, int D, bool kWide, bool kInterleaved>
__device__ inline void append_heads(const AppendArgs& a, bool values) {
  constexpr uint32_t kLanes = D / 8, kPer = 256 / kLanes;
  const uint32_t lane = threadIdx.x % kLanes, heads = a.n_heads + a.n_kv_heads * (values ? 2u : 1u);
  const uint64_t first = (uint64_t)blockIdx.x * kPer;
  const uint32_t t0 = (uint32_t)(first / heads), r = (uint32_t)(first - (uint64_t)t0 * heads) + threadIdx.x / kLanes;
  const uint32_t t = t0 + r / heads, h = r % heads;
  const bool inside = t < a.n_tok;
  const uint32_t tok = inside ? t : a.n_tok - 1u;  // (lanes past the end take part in the exchanges)
  const bool is_q = h < a.n_heads;
  const uint32_t hk = is_q ? 0u : (h - a.n_heads) % a.n_kv_heads;
  const bool is_v = h >= a.n_heads + a.n_kv_heads;
  const T* src = is_q ? static_cast<const T*>(a.q) + tok * a.q_stride + (uint64_t)h * D
                      : is_v ? static_cast<const T*>(a.v) + tok * a.v_stride + (uint64_t)hk * D
                             : static_cast<const T*>(a.k) + tok * a.k_stride + (uint64_t)hk * D;
  const auto raw = load8<T, kWide>(src + lane * 8u);
  float x[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] = (float)raw[k];
  const T* weight = static_cast<const T*>(is_q ? a.q_weight : a.k_weight);
  float sum = 0.0f;
#pragma unroll
  for (int k = 0; k < 8; ++k) sum = fmaf(x[k], x[k], sum);
#pragma unroll
  for (uint32_t d = 1; d < kLanes; d <<= 1) sum += __shfl_xor(sum, d);
  if (weight && !is_v) {
    const float by = 1.0f / sqrtf(sum * (1.0f / D) + a.eps);
    const auto w = load8<T, kWide>(weight + lane * 8u);
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
          const float u = x[2 * k], w = x[2 * k + 1];
          x[2 * k] = u * c[k] - w * s[k];
          x[2 * k + 1] = w * c[k] + u * s[k];
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
  if (!inside) return;
  if (is_q) {
    store8<T, kWide>(static_cast<T*>(a.q_out) + tok * a.q_out_stride + (uint64_t)h * D + lane * 8u, narrow8<T>(x));
    return;
  }
  const int64_t slot = a.slot[tok];
  if (slot < 0) return;
  if ((uint64_t)slot >= a.n_slots) {
    if (lane == 0) raise(a.status, MAASO_INST_BAD_PAGE);
    return;
  }
  const uint64_t page = (uint64_t)slot >> a.page_log2;
  const uint32_t place = (uint32_t)slot & ((1u << a.page_log2) - 1u);
  if (is_v) {
    C* to = reinterpret_cast<C*>(a.v_pages) + page * a.page_stride + (((uint64_t)hk * D + lane * 8u) << a.page_log2) + place;
    const float scale = sizeof(C) == 1 && a.v_scale ? a.v_scale[hk] : 1.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) store_one<T, C>(to + ((uint64_t)k << a.page_log2), raw[k], scale);
    return;
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

// Values of many tokens: a block turns 64 tokens by 64 elements of a head through shared memory.  Up to eight tokens
// that follow each other within eight places of a page are one store of eight elements, others go one by one.
constexpr uint32_t kTurnTokens = 64, kTurnPad = 66;

template <typename T, typename C, int D, bool kWide>
__device__ inline void append_values(const AppendArgs& a, uint32_t block) {
  __shared__ T tile[kTurnTokens * kTurnPad];
  const uint32_t per_token = a.n_kv_heads * (D / 64);
  const uint32_t t0 = block / per_token * kTurnTokens, hd = block % per_token;
  const uint32_t hk = hd / (D / 64), d0 = hd % (D / 64) * 64u;
  const uint32_t n = a.n_tok - t0 < kTurnTokens ? a.n_tok - t0 : kTurnTokens;
  for (uint32_t e = threadIdx.x; e < n * 8u; e += 256u) {
    const uint32_t t = e / 8u, d = e % 8u * 8u;
    const auto x = load8<T, kWide>(static_cast<const T*>(a.v) + (t0 + t) * a.v_stride + (uint64_t)hk * D + d0 + d);
#pragma unroll
    for (int k = 0; k < 8; ++k) tile[t * kTurnPad + d + k] = x[k];
  }
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
  int64_t slot = lane < n ? a.slot[t0 + lane] : -1;
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

template <typename T, typename C, int D, bool kWide, bool kInterleaved>
__global__ void __launch_bounds__(256) append_kernel(AppendArgs a) {
  if (blockIdx.x < a.head_blocks) append_heads<T, C, D, kWide, kInterleaved>(a, gridDim.x == a.head_blocks);
  else append_values<T, C, D, kWide>(a, blockIdx.x - a.head_blocks);
}

}  // namespace maaso
