// Logits as the next token is chosen from: penalties for what has been said, biases, temperature, a grammar's mask,
// and the token of the largest value, in one pass over the logits.  Bound by memory: the row in, the row out.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/maaso_instance.h"
#include "element_types.hpp"
#include "kv_pages_kernels.hpp"

namespace maaso {

constexpr uint32_t kLogitSlice = 8192;  // tokens of a row that a block takes: their counts fit in 32 KiB of LDS
constexpr uint32_t kLogitThreads = 512;
constexpr uint32_t kHasBias = 0x80000000u;

struct LogitsArgs {
  const void* logits;
  void* out;
  int32_t* chosen;
  uint64_t stride, out_stride;
  uint32_t n, vocab, slices, n_history, n_bias, n_mask, mask_words;
  const float* repetition;
  const float* frequency;
  const float* presence;
  const float* temperature;
  const int32_t* history;
  const int32_t* history_start;
  const int32_t* bias_token;
  const float* bias_value;
  const int32_t* bias_start;
  const uint32_t* mask;
  const int32_t* mask_row;
  unsigned long long* best;  // workspace [n][slices]
  uint32_t* status;
};

// A list's part for row r; nothing where its starts run backwards or past its end.
__device__ inline void list_part(const int32_t* start, uint32_t r, uint32_t size, uint32_t* status, uint32_t& begin, uint32_t& end) {
  begin = end = 0u;
  if (!start) return;
  const int32_t b = start[r], e = start[r + 1];
  if (b < 0 || e < b || (uint32_t)e > size) {
    if (threadIdx.x == 0) raise(status, MAASO_INST_BAD_BOUND);
    return;
  }
  begin = (uint32_t)b;
  end = (uint32_t)e;
}

// Larger values, then lower tokens, are larger keys; 0 is below every value.
__device__ inline unsigned long long choice_key(float x, uint32_t token) {
  const uint32_t u = __float_as_uint(x + 0.0f);  // (-0 is 0)
  const uint32_t ordered = u >> 31 ? ~u : u | 0x80000000u;
  return (unsigned long long)ordered << 32 | (uint32_t)~token;
}

__device__ inline unsigned long long wave_max(unsigned long long v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const unsigned long long o = __shfl_xor(v, d);
    v = o > v ? o : v;
  }
  return v;
}

template <typename T, typename O, bool kWide>
__global__ void __launch_bounds__(kLogitThreads) logits_kernel(LogitsArgs a) {
  __shared__ uint32_t count[kLogitSlice];
  __shared__ unsigned long long top[kLogitThreads / 64];
  const uint32_t row = blockIdx.x / a.slices, slice = blockIdx.x % a.slices;
  const uint32_t v0 = slice * kLogitSlice, n = a.vocab - v0 < kLogitSlice ? a.vocab - v0 : kLogitSlice;
  uint32_t hb, he, bb, be;
  list_part(a.history_start, row, a.n_history, a.status, hb, he);
  list_part(a.bias_start, row, a.n_bias, a.status, bb, be);
  const bool counts = he > hb || be > bb;
  if (counts) {
    for (uint32_t i = threadIdx.x; i < n; i += kLogitThreads) count[i] = 0u;
    __syncthreads();
    for (uint32_t i = hb + threadIdx.x; i < he; i += kLogitThreads) {
      const uint32_t v = (uint32_t)a.history[i];
      if (v - v0 < n) atomicAdd(&count[v - v0], 1u);
      else if (v >= a.vocab && slice == 0) raise(a.status, MAASO_INST_BAD_TOKEN);
    }
    for (uint32_t i = bb + threadIdx.x; i < be; i += kLogitThreads) {
      const int32_t v = a.bias_token[i];
      const bool good = v >= 0 && (uint32_t)v < a.vocab && (i == bb || a.bias_token[i - 1] < v);
      if (!good) {
        if (slice == 0) raise(a.status, MAASO_INST_BAD_TOKEN);
      } else if ((uint32_t)v - v0 < n) {
        atomicOr(&count[(uint32_t)v - v0], kHasBias);
      }
    }
    __syncthreads();
  }
  const float rep = a.repetition ? a.repetition[row] : 1.0f, freq = a.frequency ? a.frequency[row] : 0.0f;
  const float pres = a.presence ? a.presence[row] : 0.0f, temp = a.temperature ? a.temperature[row] : 1.0f;
  const uint32_t* bits = nullptr;
  if (a.mask) {
    const int32_t m = a.mask_row ? a.mask_row[row] : (int32_t)row;
    if (m >= 0 && (uint32_t)m < a.n_mask) bits = a.mask + (uint64_t)m * a.mask_words;
    else if (m >= 0 && threadIdx.x == 0) raise(a.status, MAASO_INST_BAD_ROW);
  }
  const T* in = static_cast<const T*>(a.logits) + row * a.stride + v0;
  O* out = a.out ? static_cast<O*>(a.out) + row * a.out_stride + v0 : nullptr;
  unsigned long long best = 0ull;
  for (uint32_t i0 = threadIdx.x * 8u; i0 < n; i0 += kLogitThreads * 8u) {
    const bool whole = kWide && i0 + 8u <= n;
    T raw[8];
    if (whole) {
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<u32x4*>(raw) = *reinterpret_cast<const u32x4*>(in + i0);
        *reinterpret_cast<u32x4*>(raw + 4) = *reinterpret_cast<const u32x4*>(in + i0 + 4);
      } else {
        *reinterpret_cast<u32x4*>(raw) = *reinterpret_cast<const u32x4*>(in + i0);
      }
    } else {
      for (uint32_t k = 0; k < 8u; ++k) raw[k] = i0 + k < n ? in[i0 + k] : (T)0.0f;
    }
    const uint32_t allowed = bits ? bits[(v0 + i0) / 32u] >> (i0 & 31u) : 0xffu;
    float x[8];
#pragma unroll
    for (uint32_t k = 0; k < 8u; ++k) {
      float y = (float)raw[k];
      if (counts && i0 + k < n) {
        const uint32_t c = count[i0 + k];
        if (c & ~kHasBias) {
          y = y > 0.0f ? y / rep : y * rep;
          y = y - (freq * (float)(c & ~kHasBias) + pres);
        }
        if (c & kHasBias) {
          uint32_t lo = bb, hi = be;  // the entry that holds the token (rare: the list is searched)
          while (hi - lo > 1u) {
            const uint32_t mid = (lo + hi) >> 1;
            if (a.bias_token[mid] <= (int32_t)(v0 + i0 + k)) lo = mid; else hi = mid;
          }
          if (a.bias_token[lo] == (int32_t)(v0 + i0 + k)) y = y + a.bias_value[lo];
        }
      }
      y = y / temp;
      if (!(allowed >> k & 1u)) y = -INFINITY;
      x[k] = y;
      if (i0 + k < n && y > -INFINITY) {
        const unsigned long long key = choice_key(y, v0 + i0 + k);
        best = key > best ? key : best;
      }
    }
    if (out) {
      O o[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] = (O)x[k];
      if (whole) {
        *reinterpret_cast<u32x4*>(out + i0) = *reinterpret_cast<const u32x4*>(o);
        if constexpr (sizeof(O) == 4) *reinterpret_cast<u32x4*>(out + i0 + 4) = *reinterpret_cast<const u32x4*>(o + 4);
      } else {
        for (uint32_t k = 0; k < 8u && i0 + k < n; ++k) out[i0 + k] = o[k];
      }
    }
  }
  if (!a.chosen) return;
  best = wave_max(best);
  if ((threadIdx.x & 63u) == 0) top[threadIdx.x >> 6] = best;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (uint32_t w = 1; w < kLogitThreads / 64u; ++w) best = top[w] > best ? top[w] : best;
    a.best[(uint64_t)row * a.slices + slice] = best;
  }
}

__global__ void __launch_bounds__(64) choose_kernel(const unsigned long long* best, uint32_t slices, int32_t* chosen) {
  unsigned long long top = 0ull;
  for (uint32_t s = threadIdx.x; s < slices; s += 64u) {
    const unsigned long long v = best[(uint64_t)blockIdx.x * slices + s];
    top = v > top ? v : top;
  }
  top = wave_max(top);
  if (threadIdx.x == 0) chosen[blockIdx.x] = top ? (int32_t)~(uint32_t)top : -1;
}

}  // namespace maaso
