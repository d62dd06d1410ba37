// The routing of tokens to experts: scores, the k largest of each token with their weights, and the tokens in the order of
// their experts, by whole-number counts, so that nothing depends on the order of blocks.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/maaso_instance.h"
#include "element_types.hpp"
#include "gate.hpp"
#include "lds_barrier.hpp"

namespace maaso {

struct RouteArgs {
  const void* logits;
  const float* bias;
  int32_t* expert;
  float* weight;
  int32_t* start;
  int32_t* token;
  int32_t* place;
  uint64_t stride;
  uint32_t n, n_experts, k;
  bool sigmoid, renorm;
  float scale;
  uint32_t chunks;     // of kChunk tokens
  uint32_t* counts;    // workspace [chunks][n_experts]: an expert's tokens in a chunk, then those before the chunk, from the expert's start on
};

constexpr uint32_t kChunk = 64;       // tokens whose places are worked out together
constexpr uint32_t kOneBlock = 256;   // tokens that one block does alone

__device__ inline double score64(float x, float bias) { return 1.0 / (1.0 + exp(-(double)x)) + (double)bias; }

// The experts of one token, by one wave: lane l has the logits of experts l, l + 64, ...; Per of them.
template <typename T, int Per, bool Biased>
__device__ inline void choose(const RouteArgs& a, uint32_t t) {
  const uint32_t lane = threadIdx.x & 63u;
  const T* row = static_cast<const T*>(a.logits) + t * a.stride;
  constexpr float kLow = -__builtin_huge_valf();
  float x[Per];
  double score[Per];
  float top = kLow;
#pragma unroll
  for (int i = 0; i < Per; ++i) {
    const uint32_t e = lane + 64u * i;
    x[i] = e < a.n_experts ? (float)row[e] : kLow;
    if (x[i] != x[i]) x[i] = kLow;
    x[i] = fminf(x[i], 3.40282347e38f);
    score[i] = (double)x[i];
    if constexpr (Biased) {
      if (x[i] > kLow) {
        score[i] = score64(x[i], a.bias[e]);
        if (!(score[i] > (double)kLow)) x[i] = kLow;
      }
      if (x[i] == kLow) score[i] = (double)kLow;
    }
    top = fmaxf(top, x[i]);
  }
  float total = 1.0f;
  if (!a.sigmoid) {
#pragma unroll
    for (int d = 32; d > 0; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
    total = 0.0f;
#pragma unroll
    for (int i = 0; i < Per; ++i) total += x[i] > kLow ? expf(x[i] - top) : 0.0f;
#pragma unroll
    for (int d = 32; d > 0; d /= 2) total += __shfl_xor(total, d);
  }
  float chosen = 0.0f, mine = 0.0f;
  int32_t which = -1;
  for (uint32_t j = 0; j < a.k; ++j) {
    double best = (double)kLow;
    uint32_t at = 0xffffffffu;
#pragma unroll
    for (int i = 0; i < Per; ++i) {
      if (score[i] > best) {
        best = score[i];
        at = lane + 64u * i;
      }
    }
#pragma unroll
    for (int d = 32; d > 0; d /= 2) {
      const double o = __shfl_xor(best, d);
      const uint32_t oa = (uint32_t)__shfl_xor((int)at, d);
      if (o > best || (o == best && oa < at)) {
        best = o;
        at = oa;
      }
    }
    if (at == 0xffffffffu) break;  // the same for every lane
    float p = 0.0f;
#pragma unroll
    for (int i = 0; i < Per; ++i) {
      if (at == lane + 64u * i) {
        p = a.sigmoid ? sigmoid(x[i]) : expf(x[i] - top) / total;
        score[i] = (double)kLow;
      }
    }
    p = __shfl(p, (int)(at & 63u));
    chosen += p;
    if (lane == j) {
      mine = p;
      which = (int32_t)at;
    }
  }
  if (lane < a.k) {
    const float by = a.renorm ? chosen > 0.0f ? mine / chosen : 0.0f : mine;
    a.expert[(uint64_t)t * a.k + lane] = which;
    a.weight[(uint64_t)t * a.k + lane] = which < 0 ? 0.0f : by * a.scale;
  }
}

template <typename T, int Per, bool Biased> __global__ void __launch_bounds__(256) route_choose_kernel(RouteArgs a) {
  const uint32_t t = blockIdx.x * 4u + threadIdx.x / 64u;
  if (t < a.n) choose<T, Per, Biased>(a, t);
}

// Which tokens of the chunk go to each expert, a bit each: an expert is chosen by a token once at most, so a token's rank among its
// expert's is the number of bits below its own.  bits: [n_experts][words].
__device__ inline void mark_chosen(const RouteArgs& a, uint32_t first, uint32_t tokens, uint32_t* bits, uint32_t words) {
  for (uint32_t i = threadIdx.x; i < a.n_experts * words; i += blockDim.x) bits[i] = 0u;
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < tokens * a.k; i += blockDim.x) {
    const int32_t e = a.expert[(uint64_t)first * a.k + i];
    const uint32_t t = i / a.k;
    if (e >= 0) atomicOr(&bits[(uint32_t)e * words + t / 32u], 1u << (t & 31u));
  }
  lds_atomics_barrier();
}

__device__ inline void put_chosen(const RouteArgs& a, uint32_t first, uint32_t tokens, const uint32_t* bits, uint32_t words, const uint32_t* before) {
  for (uint32_t i = threadIdx.x; i < tokens * a.k; i += blockDim.x) {
    const int32_t e = a.expert[(uint64_t)first * a.k + i];
    const uint32_t t = i / a.k;
    int32_t to = -1;
    if (e >= 0) {
      const uint32_t* b = bits + (uint32_t)e * words;
      uint32_t rank = before[e] + (uint32_t)__builtin_popcount(b[t / 32u] & ((1u << (t & 31u)) - 1u));
      for (uint32_t w = 0; w < t / 32u; ++w) rank += (uint32_t)__builtin_popcount(b[w]);
      to = (int32_t)rank;
      a.token[rank] = (int32_t)(first + t);
    }
    a.place[(uint64_t)first * a.k + i] = to;
  }
}

// An exclusive sum over up to 1024 threads' values; the sum of all goes to `all`.
__device__ inline uint32_t block_before(uint32_t v, uint32_t* meet, uint32_t& all) {
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x / 64u;
  uint32_t upto = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t o = (uint32_t)__shfl_up((int)upto, d);
    upto += (int)lane >= d ? o : 0u;
  }
  if (lane == 63u) meet[wave] = upto;
  __syncthreads();
  uint32_t below = 0u;
  all = 0u;
  for (uint32_t w = 0; w < blockDim.x / 64u; ++w) {
    below += w < wave ? meet[w] : 0u;
    all += meet[w];
  }
  return below + upto - v;
}

// Few tokens: chosen and put in order by one block.  dynamic: bits [n_experts][words], before [n_experts]
__global__ void __launch_bounds__(1024) route_order_kernel(RouteArgs a) {
  extern __shared__ uint32_t room[];
  __shared__ uint32_t meet[16];
  const uint32_t words = (a.n + 31u) / 32u;
  uint32_t* before = room + a.n_experts * words;
  mark_chosen(a, 0u, a.n, room, words);
  uint32_t mine = 0u, all;
  if (threadIdx.x < a.n_experts) {
    for (uint32_t w = 0; w < words; ++w) mine += (uint32_t)__builtin_popcount(room[threadIdx.x * words + w]);
  }
  const uint32_t at = block_before(mine, meet, all);
  if (threadIdx.x < a.n_experts) {
    before[threadIdx.x] = at;
    a.start[threadIdx.x] = (int32_t)at;
  }
  if (threadIdx.x == 0u) a.start[a.n_experts] = (int32_t)all;
  __syncthreads();
  put_chosen(a, 0u, a.n, room, words, before);
  for (uint32_t i = all + threadIdx.x; i < a.n * a.k; i += 1024u) a.token[i] = -1;
}

__global__ void __launch_bounds__(256) route_count_kernel(RouteArgs a) {
  extern __shared__ uint32_t room[];
  const uint32_t first = blockIdx.x * kChunk, tokens = min(kChunk, a.n - first), words = kChunk / 32u;
  mark_chosen(a, first, tokens, room, words);
  for (uint32_t e = threadIdx.x; e < a.n_experts; e += 256u)
    a.counts[(uint64_t)blockIdx.x * a.n_experts + e] = (uint32_t)__builtin_popcount(room[e * words]) + (uint32_t)__builtin_popcount(room[e * words + 1u]);
}

// One block: the experts' starts, and each chunk's before it.
__global__ void __launch_bounds__(1024) route_starts_kernel(RouteArgs a) {
  __shared__ uint32_t meet[16];
  uint32_t mine = 0u, all;
  const uint32_t e = threadIdx.x;
  if (e < a.n_experts) {
    for (uint32_t c = 0; c < a.chunks; ++c) mine += a.counts[(uint64_t)c * a.n_experts + e];
  }
  uint32_t at = block_before(mine, meet, all);
  if (e < a.n_experts) {
    a.start[e] = (int32_t)at;
    for (uint32_t c = 0; c < a.chunks; ++c) {
      const uint64_t i = (uint64_t)c * a.n_experts + e;
      const uint32_t n = a.counts[i];
      a.counts[i] = at;
      at += n;
    }
  }
  if (e == 0u) a.start[a.n_experts] = (int32_t)all;
}

__global__ void __launch_bounds__(256) route_place_kernel(RouteArgs a) {
  extern __shared__ uint32_t room[];
  const uint32_t first = blockIdx.x * kChunk, tokens = min(kChunk, a.n - first), words = kChunk / 32u;
  mark_chosen(a, first, tokens, room, words);
  put_chosen(a, first, tokens, room, words, a.counts + (uint64_t)blockIdx.x * a.n_experts);
  const uint32_t all = (uint32_t)a.start[a.n_experts];
  for (uint32_t i = first * a.k + threadIdx.x; i < (first + tokens) * a.k; i += 256u)
    if (i >= all) a.token[i] = -1;
}

}  // namespace maaso
