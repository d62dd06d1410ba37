// Rows of activations to 8-bit integers with a scale each, behind a norm or a gate; and the joining of experts' rows.
// Both are bound by memory: 8192 rows of 4096, 16 bits, 20.8 us, 4.85 TB/s, what a large copy reaches; with a norm 25, for its weight comes from
// the cache for each row; the gate (4096 rows of 2 x 8192) 36, 4.6 TB/s.  8192 tokens' eight rows of 4096, joined, 144.5 us, 4.65 TB/s.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/maaso_instance.h"
#include "element_types.hpp"
#include "gate.hpp"

namespace maaso {

struct QuantizeArgs {
  const void* x;
  const void* weight;
  int8_t* q;
  float* scale;
  uint64_t x_stride, q_stride;  // elements
  uint32_t n, width;
  float eps;
};

// Eight elements that begin anywhere.
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Eight { T v[8]; };

// Elements [at, at + 8) of a row of `width`, zeros from its end on.
template <typename T> __device__ inline void load8(const T* row, uint32_t at, uint32_t width, float (&y)[8]) {
  if (at + 8u <= width) {
    const Eight<T> e = *reinterpret_cast<const Eight<T>*>(row + at);
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = (float)e.v[k];
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = at + (uint32_t)k < width ? (float)row[at + k] : 0.0f;
  }
}

// Registers hold no more than a row needs (4096 with a norm: two turns 25.0 us, room for four 29.4), and a block takes one row: blocks that take
// one after the other, the next one's loads under way, have fewer beside them and were slower (31.7).
// One row to `Threads` threads, eight neighbouring elements of each in turn, the first Held turns in registers; what is
// longer is read, and its gate worked out, a second time.  One reduction: with a norm, max |x * weight| and the sum of squares are
// taken together, for y = (x * weight) / sqrt(...) is largest where x * weight is.
template <typename T, int Form, int Threads, int Held>
__global__ void __launch_bounds__(Threads == 64 ? 256 : Threads) quantize_kernel(QuantizeArgs a) {
  constexpr int kRows = Threads == 64 ? 4 : 1, kWaves = Threads / 64;  // rows of a block, waves of a row
  __shared__ float sums[kWaves];
  __shared__ uint32_t tops[kWaves];
  const uint32_t thread = threadIdx.x % Threads, row = blockIdx.x * kRows + threadIdx.x / Threads;
  if (row >= a.n) return;  // (a whole wave, or a whole block)
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  const T* weight = static_cast<const T*>(a.weight);
  const uint32_t turns = (a.width + 8u * Threads - 1u) / (8u * Threads);

  constexpr uint32_t kInfinite = 0x7f800000u;
  float sum = 0.0f;
  uint32_t top = 0u;  // of the magnitudes' bits: an infinity is above every number, a NaN above that
  auto values = [&](uint32_t turn, float (&y)[8], bool first) {
    const uint32_t at = (turn * Threads + thread) * 8u;
    load8(x, at, a.width, y);
    if constexpr (Form == MAASO_ROWS_NORM) {
      if (first) {
#pragma unroll
        for (int k = 0; k < 8; ++k) sum = fmaf(y[k], y[k], sum);
      }
      if (weight) {
        float w[8];
        load8(weight, at, a.width, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] *= w[k];
      }
    } else if constexpr (Form == MAASO_ROWS_GATED) {
      float up[8];
      load8(x + a.width, at, a.width, up);
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = silu(y[k]) * up[k];
    }
    if (first) {
#pragma unroll
      for (int k = 0; k < 8; k += 2)
        top = max(max(__builtin_bit_cast(uint32_t, y[k]) & 0x7fffffffu, __builtin_bit_cast(uint32_t, y[k + 1]) & 0x7fffffffu), top);
    }
  };
  float held[Held][8];
#pragma unroll
  for (int h = 0; h < Held; ++h) {
    if ((uint32_t)h < turns) values(h, held[h], true);
  }
  for (uint32_t t = Held; t < turns; ++t) {
    float y[8];
    values(t, y, true);
  }
  auto meet = [&](bool again) {  // sum and top over the row's threads
#pragma unroll
    for (int d = 32; d > 0; d /= 2) {
      if constexpr (Form == MAASO_ROWS_NORM) sum += __shfl_xor(sum, d);
      top = max(top, (uint32_t)__shfl_xor((int)top, d));
    }
    if constexpr (kWaves > 1) {
      if (again) __syncthreads();  // the last results have been read
      if ((thread & 63u) == 0u) {
        sums[thread / 64u] = sum;
        tops[thread / 64u] = top;
      }
      __syncthreads();
      sum = 0.0f;
      top = 0u;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        sum += sums[w];
        top = max(top, tops[w]);
      }
    }
  };
  meet(false);
  bool good = top < kInfinite, apart = false;
  float by = 1.0f, lift = 1.0f;
  // A row apart (the same for all of its threads): squares or products of numbers are beyond binary32, or below what it holds whole, and the
  // normed numbers need not be.  It is read again, in the order of the formula: the squares' sum, of numbers raised by 2^100 where it was next to
  // nothing and eps does not outweigh that, and then (x / sqrt(...)) * weight, which is worked out once more where it is stored.  (8000 rows of 4096
  // numbers of 1e-25 with eps 0 41.7 us, of zeros 31.2, of others 25.5, 25.3 without this.)
  auto normed = [&](uint32_t turn, float (&y)[8]) {
    const uint32_t at = (turn * Threads + thread) * 8u;
    load8(x, at, a.width, y);
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = y[k] * lift * by;
    if (weight) {
      float w[8];
      load8(weight, at, a.width, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] *= w[k];
    }
  };
  if constexpr (Form == MAASO_ROWS_NORM) {
    const bool finite = __builtin_bit_cast(uint32_t, sum) < kInfinite, faint = sum < 0x1p-90f && a.eps < 0x1p-60f;
    good = good && finite;
    apart = finite && (faint || top == kInfinite || top < __builtin_bit_cast(uint32_t, 0x1p-100f));
    if (apart) {
      if (faint) {
        lift = 0x1p100f;
        sum = 0.0f;
        for (uint32_t t = 0; t < turns; ++t) {
          float y[8];
          load8(x, (t * Threads + thread) * 8u, a.width, y);
#pragma unroll
          for (int k = 0; k < 8; ++k) sum = fmaf(y[k] * lift, y[k] * lift, sum);
        }
        top = 0u;
        meet(true);
      }
      const double mean = (double)sum / (double)a.width * (faint ? 0x1p-200 : 1.0) + (double)a.eps;
      by = mean > 0.0 ? (float)(1.0 / sqrt(mean) * (faint ? 0x1p-100 : 1.0)) : 0.0f;
      sum = 0.0f;
      top = 0u;
      for (uint32_t t = 0; t < turns; ++t) {
        float y[8];
        normed(t, y);
#pragma unroll
        for (int k = 0; k < 8; ++k) top = max(top, __builtin_bit_cast(uint32_t, y[k]) & 0x7fffffffu);
      }
      meet(true);
      good = top < kInfinite;
    }
  }
  float most = __builtin_bit_cast(float, top);
  if constexpr (Form == MAASO_ROWS_NORM) {
    if (good && top && !apart) {
      by = 1.0f / sqrtf(sum / (float)a.width + a.eps);
      most *= by;
      good = most < __builtin_huge_valf();
    }
  }
  if (thread == 0u) a.scale[row] = good ? most / 127.0f : __builtin_nanf("");
  // Rows of very small numbers are raised by 2^100 first: 1 / m would be no number for them.
  const float raise = most < 0x1p-100f ? 0x1p100f : 1.0f, per = good && most > 0.0f ? 1.0f / (most * raise) * 127.0f : 0.0f;
  int8_t* q = a.q + row * a.q_stride;
  // Added to 1.5 * 2^23 a number up to 2^22 is rounded to a whole one, ties to even, whose lowest byte is the sum's.  (The
  // reciprocal and both products are rounded to binary32 first, as the interface has it: whoever brings a row as it is to 8 bits in binary32 gets
  // the same bytes.  Behind a norm or a gate y is binary32 in this kernel's own order.  Of 32.8 million bytes behind a norm 47 to 233 were not
  // those of 64 bits, numbers halfway between two bytes nearly all, of the formula in torch's binary32 51 to 252.)
  auto store = [&](uint32_t turn, float (&y)[8], float by) {
    constexpr float kWhole = 12582912.0f;
    const uint32_t at = (turn * Threads + thread) * 8u;
    uint32_t b[2] = {0u, 0u};
    if (per != 0.0f) {  // (the same for the row)
      if (raise != 1.0f) {
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] *= raise;
      }
      uint32_t v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = __builtin_bit_cast(uint32_t, (Form == MAASO_ROWS_NORM ? y[k] * by * per : y[k] * per) + kWhole);
#pragma unroll
      for (int h = 0; h < 2; ++h)
        b[h] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(v[4 * h + 3], v[4 * h + 2], 0x0c0c0400u), __builtin_amdgcn_perm(v[4 * h + 1], v[4 * h], 0x0c0c0400u), 0x05040100u);
    }
    if (at + 8u <= a.width) {
      *reinterpret_cast<u32x2*>(q + at) = (u32x2){b[0], b[1]};
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (at + (uint32_t)k < a.width) q[at + k] = (int8_t)(b[k / 4] >> (8 * (k % 4)));
    }
  };
  if constexpr (Form == MAASO_ROWS_NORM) {
    if (apart) {
      for (uint32_t t = 0; t < turns; ++t) {
        float y[8] = {};
        if (per != 0.0f) normed(t, y);
        store(t, y, 1.0f);
      }
      return;
    }
  }
#pragma unroll
  for (int h = 0; h < Held; ++h) {
    if ((uint32_t)h < turns) store(h, held[h], by);
  }
  for (uint32_t t = Held; t < turns; ++t) {
    float y[8];
    values(t, y, false);
    store(t, y, by);
  }
}

struct CombineArgs {
  const void* y;
  const void* residual;
  void* out;
  const int32_t* place;
  const float* weight;
  uint64_t y_stride, residual_stride, out_stride;  // elements
  uint32_t n, k, width, n_rows;
  uint32_t* status;
};

template <typename T> __device__ inline void store8(T* row, uint32_t at, uint32_t width, const float (&y)[8]) {
  if constexpr (sizeof(T) == 4) {
    if (at + 8u <= width) {
      Eight<T> e;
#pragma unroll
      for (int k = 0; k < 8; ++k) e.v[k] = y[k];
      *reinterpret_cast<Eight<T>*>(row + at) = e;
      return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (at + (uint32_t)k < width) row[at + k] = y[k];
  } else {
    const auto v = narrow8<T>(y);
    if (at + 8u <= width) {
      *reinterpret_cast<Eight<T>*>(row + at) = __builtin_bit_cast(Eight<T>, v);
      return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (at + (uint32_t)k < width) row[at + k] = v[k];
  }
}

// A thread is eight neighbouring elements of a token; the token's rows are read four at a time, for loads under way are what it waits for.
template <typename T> __global__ void __launch_bounds__(256) combine_kernel(CombineArgs a) {
  const uint32_t per = (a.width + 7u) / 8u;
  const uint64_t at = (uint64_t)blockIdx.x * 256u + threadIdx.x;
  const uint64_t token = at / per;
  const uint32_t col = (uint32_t)(at - token * per) * 8u;
  if (token >= a.n) return;
  float sum[8] = {};
  if (a.residual) load8(static_cast<const T*>(a.residual) + token * a.residual_stride, col, a.width, sum);
  for (uint32_t j = 0; j < a.k; j += 4u) {
    float y[4][8], w[4];
#pragma unroll
    for (uint32_t u = 0; u < 4u; ++u) {
      const bool in = j + u < a.k;
      const int32_t p = in ? a.place[token * a.k + j + u] : -1;
      const bool there = (uint32_t)p < a.n_rows;
      if (p >= 0 && !there) atomicOr(a.status, MAASO_INST_BAD_ROW);
      w[u] = there ? a.weight ? a.weight[token * a.k + j + u] : 1.0f : 0.0f;
      if (there) {
        load8(static_cast<const T*>(a.y) + (uint64_t)(uint32_t)p * a.y_stride, col, a.width, y[u]);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) y[u][k] = 0.0f;
      }
    }
#pragma unroll
    for (uint32_t u = 0; u < 4u; ++u)
#pragma unroll
      for (int k = 0; k < 8; ++k) sum[k] = fmaf(w[u], y[u][k], sum[k]);
  }
  store8(static_cast<T*>(a.out) + token * a.out_stride, col, a.width, sum);
}

}  // namespace maaso
