// Logits as the next token is chosen from: penalties for what has been said, biases, temperature, a grammar's mask,
// and the token of the largest value, in one pass over the logits.  Bound by memory, the row in, the row out, and by the
// instructions of tokens that the history or a bias marks: 192 rows of 131,072 (16 bits in, 32 out, half of them masked) in
// 43 us, 3.6 TB/s; one row of 50,257 in 7.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/maaso_instance.h"
#include "element_types.hpp"
#include "kv_pages_kernels.hpp"
#include "lds_barrier.hpp"

namespace maaso {

// A block takes a slice of a row, kPieces times eight neighbouring tokens a thread: 4096 tokens where there are rows enough
// to fill the card (their marks are 16 KiB of LDS, eight blocks to a compute unit), 1024 where there are few.  The 192 rows 43.1 us;
// with 8192 tokens a block of 512 threads 43.1, of 256 threads 48.0, with 2048 tokens 43.7.  One row of 50,257 in 1024 a block,
// without the second launch, 7.0 for 9.0.
constexpr uint32_t kManyThreads = 256, kManyPieces = 2, kFewThreads = 128, kFewPieces = 1;
constexpr uint32_t kManySlice = 8u * kManyThreads * kManyPieces, kFewSlice = 8u * kFewThreads * kFewPieces;
// Outputs of more than 8 MiB whose rows begin at multiples of 16 bytes are written past the caches: the 192 rows 50 to 43 us, 18 rows
// of 131,072 10.2 to 9.6; 5 rows 7.1 to 7.3, and 126 rows of 100,003 16-bit logits, whose pieces lie across lines, 21.5 to 23.5.
constexpr uint64_t kLogitPast = 8u << 20;
constexpr uint32_t kFewRows = 1024;  // rows that the instance keeps a LogitsRow for
// A token's mark: how often the history has it, and above kCountBits the number of its bias among the row's, from 1 on.  Rows
// of a longer history or more biases mark a bias by the highest bit alone, and search for it.
constexpr uint32_t kCountBits = 20, kListed = 512;
constexpr uint32_t kHasBias = 0x80000000u;

// A row's largest key and how many of its slices are done; zeros between calls.  Rows have cache lines of their own.
struct __attribute__((aligned(128))) LogitsRow {
  unsigned long long key;
  uint32_t done;
};

// Eight elements at any alignment of an element's: 16-byte accesses all the same.
template <typename T> struct __attribute__((packed, aligned(2))) Piece { T v[8]; };

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
  bool past;                 // what is written goes past the caches
  unsigned long long* best;  // workspace [n][slices], many rows
  LogitsRow* meet;           // [n], few rows
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

// y / b rounded once, for eight values, with r = 1 / b rounded once: two corrections of y r by the remainder, which a fused
// multiply-add gives exactly; the first brings the quotient within one unit of its last place, from where the second rounds
// it as a division would (Markstein, IBM J. Res. Dev. 34, 1990).  Five operations instead of the division's eleven or so.
// Magnitudes for which a product or remainder could leave the normal range, zeros, infinities and NaN are divided.
__device__ inline void divide8(float (&y)[8], float b, float r) {
  float low = fabsf(y[0]), high = low, sum = y[0];
#pragma unroll
  for (int k = 1; k < 8; ++k) {
    low = fminf(low, fabsf(y[k]));
    high = fmaxf(high, fabsf(y[k]));
    sum += y[k];  // (NaN if one is: minimum and maximum pass over it)
  }
  if (low >= 0x1p-60f && high <= 0x1p60f && sum == sum) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float q = y[k] * r;
      q = fmaf(fmaf(-q, b, y[k]), r, q);
      y[k] = fmaf(fmaf(-q, b, y[k]), r, q);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = y[k] / b;
  }
}

template <typename T, typename O, uint32_t kThreads, uint32_t kPieces>
__global__ void __launch_bounds__(kThreads) logits_kernel(LogitsArgs a) {
  constexpr uint32_t kSlice = 8u * kThreads * kPieces;
  __shared__ __align__(16) uint32_t mark[kSlice];
  __shared__ float bias[kListed];
  __shared__ unsigned long long top[kThreads / 64];
  const uint32_t row = blockIdx.x / a.slices, slice = blockIdx.x % a.slices;
  const uint32_t v0 = slice * kSlice, n = a.vocab - v0 < kSlice ? a.vocab - v0 : kSlice;
  // The logits are asked for first, and come while the row's history is counted.
  const T* in = static_cast<const T*>(a.logits) + row * a.stride + v0;
  Piece<T> raw[kPieces];
#pragma unroll
  for (uint32_t p = 0; p < kPieces; ++p) {
    const uint32_t i0 = (p * kThreads + threadIdx.x) * 8u;
    if (i0 + 8u <= n) {
      raw[p] = *reinterpret_cast<const Piece<T>*>(in + i0);
    } else {
#pragma unroll
      for (uint32_t k = 0; k < 8u; ++k) raw[p].v[k] = i0 + k < n ? in[i0 + k] : (T)0.0f;
    }
  }
  uint32_t hb, he, bb, be;
  list_part(a.history_start, row, a.n_history, a.status, hb, he);
  list_part(a.bias_start, row, a.n_bias, a.status, bb, be);
  const float rep = a.repetition ? a.repetition[row] : 1.0f, freq = a.frequency ? a.frequency[row] : 0.0f;
  const float pres = a.presence ? a.presence[row] : 0.0f, temp = a.temperature ? a.temperature[row] : 1.0f;
  const uint32_t* bits = nullptr;
  if (a.mask) {
    const int32_t m = a.mask_row ? a.mask_row[row] : (int32_t)row;
    if (m >= 0 && (uint32_t)m < a.n_mask) bits = a.mask + (uint64_t)m * a.mask_words;
    else if (m >= 0 && threadIdx.x == 0) raise(a.status, MAASO_INST_BAD_ROW);
  }
  const bool counts = he > hb || be > bb, listed = he - hb < 1u << kCountBits && be - bb <= kListed;
  if (counts) {
#pragma unroll
    for (uint32_t i = 0; i < kSlice / 4u; i += kThreads) reinterpret_cast<u32x4*>(mark)[i + threadIdx.x] = (u32x4){0u, 0u, 0u, 0u};
    __syncthreads();
    for (uint32_t i0 = hb + threadIdx.x; i0 < he; i0 += 4u * kThreads) {  // (he <= 2^31 - 1)
      uint32_t v[4];
#pragma unroll
      for (uint32_t k = 0; k < 4u; ++k) v[k] = i0 + k * kThreads < he ? (uint32_t)a.history[i0 + k * kThreads] : v0;
#pragma unroll
      for (uint32_t k = 0; k < 4u; ++k) {
        if (i0 + k * kThreads >= he) break;
        if (v[k] - v0 < n) atomicAdd(&mark[v[k] - v0], 1u);
        else if (v[k] >= a.vocab && slice == 0) raise(a.status, MAASO_INST_BAD_TOKEN);
      }
    }
    for (uint32_t i = bb + threadIdx.x; i < be; i += kThreads) {
      const int32_t v = a.bias_token[i];
      const bool good = v >= 0 && (uint32_t)v < a.vocab && (i == bb || a.bias_token[i - 1] < v);
      if (listed) bias[i - bb] = a.bias_value[i];
      if (!good) {
        if (slice == 0) raise(a.status, MAASO_INST_BAD_TOKEN);
      } else if ((uint32_t)v - v0 < n) {
        // (a token listed twice, out of order, is marked by ones: a number that no bias has)
        const uint32_t old = atomicOr(&mark[(uint32_t)v - v0], listed ? (i - bb + 1u) << kCountBits : kHasBias);
        if (listed && old >> kCountBits) atomicOr(&mark[(uint32_t)v - v0], ~0u << kCountBits);
      }
    }
    lds_atomics_barrier();
  }
  const bool quick = temp >= 0x1p-30f && temp <= 0x1p30f;
  const float inverse = 1.0f / temp;
  O* out = a.out ? static_cast<O*>(a.out) + row * a.out_stride + v0 : nullptr;
  float best = -INFINITY;
  uint32_t best_at = 0xffffffffu;  // (none)
#pragma unroll
  for (uint32_t p = 0; p < kPieces; ++p) {
    const uint32_t i0 = (p * kThreads + threadIdx.x) * 8u;
    if (i0 >= n) break;
    float x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = (float)raw[p].v[k];
    if (counts) {
      const u32x4 c0 = *reinterpret_cast<const u32x4*>(mark + i0), c1 = *reinterpret_cast<const u32x4*>(mark + i0 + 4);
      if ((c0[0] | c0[1] | c0[2] | c0[3] | c1[0] | c1[1] | c1[2] | c1[3]) != 0u) {
#pragma unroll
        for (uint32_t k = 0; k < 8u; ++k) {
          const uint32_t c = k < 4u ? c0[k & 3u] : c1[k & 3u], times = c & (listed ? (1u << kCountBits) - 1u : ~kHasBias);
          float y = x[k];
          if (times) {
            y = y > 0.0f ? y / rep : y * rep;
            y = y - (freq * (float)times + pres);
          }
          if (c != times) {
            if (listed) {
              const uint32_t at = c >> kCountBits;
              if (at <= kListed) y = y + bias[at - 1u];
            } else {
              uint32_t lo = bb, hi = be;  // the entry that holds the token
              while (hi - lo > 1u) {
                const uint32_t mid = (lo + hi) >> 1;
                if (a.bias_token[mid] <= (int32_t)(v0 + i0 + k)) lo = mid; else hi = mid;
              }
              if (a.bias_token[lo] == (int32_t)(v0 + i0 + k)) y = y + a.bias_value[lo];
            }
          }
          x[k] = y;
        }
      }
    }
    if (quick && temp != 1.0f) {
      divide8(x, temp, inverse);
    } else if (temp != 1.0f) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = x[k] / temp;
    }
    const uint32_t allowed = bits ? bits[(v0 + i0) / 32u] >> (i0 & 31u) : 0xffu;
#pragma unroll
    for (uint32_t k = 0; k < 8u; ++k) {
      if (!(allowed >> k & 1u)) x[k] = -INFINITY;
      if (x[k] > best && i0 + k < n) {  // (ascending tokens: the lowest of equals stays)
        best = x[k];
        best_at = v0 + i0 + k;
      }
    }
    if (out) {
      Piece<O> o;
#pragma unroll
      for (int k = 0; k < 8; ++k) o.v[k] = (O)x[k];
      if (i0 + 8u <= n) {
        if (a.past) {
          typedef uint32_t sixteen __attribute__((ext_vector_type(4), aligned(2)));
          keep_apart();
#pragma unroll
          for (uint32_t w = 0; w < sizeof(O) / 2u; ++w)
            __builtin_nontemporal_store(reinterpret_cast<const sixteen*>(&o)[w], reinterpret_cast<sixteen*>(out + i0) + w);
          keep_apart();
        } else {
          *reinterpret_cast<Piece<O>*>(out + i0) = o;
        }
      } else {
#pragma unroll
        for (uint32_t k = 0; k < 8u; ++k)
          if (i0 + k < n) out[i0 + k] = o.v[k];
      }
    }
  }
  if (!a.chosen) return;
  unsigned long long key = wave_max(best_at == 0xffffffffu ? 0ull : choice_key(best, best_at));
  if ((threadIdx.x & 63u) == 0) top[threadIdx.x >> 6] = key;
  __syncthreads();
  if (threadIdx.x != 0) return;
#pragma unroll
  for (uint32_t w = 1; w < kThreads / 64u; ++w) key = top[w] > key ? top[w] : key;
  if (!a.meet) {
    a.best[(uint64_t)row * a.slices + slice] = key;
    return;
  }
  // The row's last slice writes the choice and leaves zeros.  What is known here of another slice's key is known by atomics
  // alone: each has had its old value back, so is done, before its block counts itself.
  LogitsRow* m = a.meet + row;
  unsigned long long old = atomicMax(&m->key, key);
  asm volatile("" : "+v"(old)::"memory");
  __builtin_amdgcn_s_waitcnt(0);
  if (atomicAdd(&m->done, 1u) == a.slices - 1u) {
    key = atomicExch(&m->key, 0ull);
    atomicExch(&m->done, 0u);
    a.chosen[row] = key ? (int32_t)~(uint32_t)key : -1;
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
