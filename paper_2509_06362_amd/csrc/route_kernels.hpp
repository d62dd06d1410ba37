// The routing of tokens to experts: scores, the k largest of each token with their weights, and the tokens in the order of
// their experts, by whole-number counts, so that nothing depends on the order of blocks.  Bound by instructions: a round of the choice is
// some 160 for four tokens.  64 tokens of 64 experts, 6 chosen, 5.2 us, one launch; 16384 tokens of 256, 8 chosen, with a bias, 24: choosing 14.6,
// counts 5.2, places 4.2 (a wave to a token, double precision throughout: 124).
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
  uint32_t chunks;   // of kChunk tokens
  uint32_t* before;  // workspace [chunks][n_experts]: an expert's tokens in a chunk, then those of the chunks before it
  uint32_t* total;   // workspace [n_experts]
};

constexpr uint32_t kChunk = 64;      // tokens whose places are worked out together
constexpr uint32_t kOneBlock = 64;   // tokens by quads held that one block chooses for and puts in order alone
constexpr uint32_t kOrderTokens = 512, kOrderChoices = 2560, kOrderRoom = 48u << 10;  // that one block puts in order; bytes of shared memory

// Every control used here reads a lane that is there.
template <int Ctrl> __device__ inline uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, Ctrl, 0xf, 0xf, true); }
template <int Ctrl> __device__ inline float dpp(float v) { return __builtin_bit_cast(float, dpp<Ctrl>(__builtin_bit_cast(uint32_t, v))); }

// Over groups of Lanes neighbouring lanes (16, 32 or 64); every lane ends with the group's value.
template <int Lanes, typename V, typename Op> __device__ inline V join(V v, Op op) {
  v = op(v, dpp<0xb1>(v));   // lane ^ 1
  v = op(v, dpp<0x4e>(v));   // lane ^ 2
  v = op(v, dpp<0x141>(v));  // the mirrored half of eight
  v = op(v, dpp<0x140>(v));  // the mirrored sixteen
  if constexpr (Lanes >= 32) v = op(v, (V)__shfl_xor(v, 16));
  if constexpr (Lanes >= 64) v = op(v, (V)__shfl_xor(v, 32));
  return v;
}
template <int Lanes> __device__ inline uint32_t largest(uint32_t v) {
  return join<Lanes>(v, [](uint32_t a, uint32_t b) { return max(a, b); });
}
template <int Lanes> __device__ inline uint32_t lowest(uint32_t v) {
  return join<Lanes>(v, [](uint32_t a, uint32_t b) { return min(a, b); });
}
template <int Lanes> __device__ inline float in_all(float v) {
  return join<Lanes>(v, [](float a, float b) { return a + b; });
}

// A score as a whole number that is larger where the score is; 0, which none has, is below them all.  (0 is added: -0 is 0.)
__device__ inline uint32_t key_of(float s) {
  const uint32_t b = __builtin_bit_cast(uint32_t, s + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ inline float score_of(uint32_t key) { return __builtin_bit_cast(float, key ^ ((uint32_t)((int32_t)~key >> 31) | 0x80000000u)); }

constexpr float kNever = -__builtin_huge_valf();  // the score of what is not chosen, or has been
constexpr float kNoShare = -690.0f;               // a sigmoid of what is below it, 2^-995, counts as 0

__device__ inline double score64(float x, float bias) { return 1.0 / (1.0 + exp(-(double)x)) + (double)bias; }

// Four neighbouring logits that begin anywhere.
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Four { T v[4]; };

// The experts of one token, by Lanes lanes that hold 4 Quads scores each; lane l those of experts 4 l + 4 Lanes q + c.  A round
// takes the largest score, then the lowest expert that has it.  Scores with a bias are compared in 64 bits: they are worked out in
// 32, which is wrong by 2^-22 + 2^-24 |score| at most.  Where two that follow each other are within 2^-21 (1 + |score|) of each
// other, those taken, and as many more as follow so closely, are put in order in 64 bits, a lane to each; where there are more of them
// than lanes' places, every round is gone through again in 64.
template <typename T, int Lanes, int Quads, bool Biased> struct Chooser {
  static constexpr int kHeld = 4 * Quads, kSlots = Lanes >= 32 ? 1 : 2;
  uint32_t lane;
  const T* row;
  int32_t which[kSlots];  // choices lane, lane + Lanes
  uint32_t rank[kSlots];  // where they stand

  __device__ inline uint32_t expert(int i) const { return 4u * lane + 4u * Lanes * (uint32_t)(i / 4) + (uint32_t)(i % 4); }
  static __device__ inline float tidy(float x) { return fminf(x != x ? kNever : x, 3.40282347e38f); }
  __device__ inline float logit(int32_t e) const { return tidy((float)row[e < 0 ? 0 : e]); }

  __device__ inline void keep(uint32_t j, uint32_t at) {
#pragma unroll
    for (int h = 0; h < kSlots; ++h) which[h] = j == lane + (uint32_t)(h * Lanes) ? (int32_t)at : which[h];
  }

  // The rounds by keys s.  With a bias: true where all of them would have to be in 64 bits.
  __device__ inline bool rounds(uint32_t k, const float* bias, uint32_t (&s)[kHeld]) {
    bool near = false, full = false;
    float before = __builtin_huge_valf();
    uint32_t j = 0;
    for (; Biased || j < k; ++j) {
      uint32_t m = s[0];
#pragma unroll
      for (int i = 1; i + 1 < kHeld; i += 2) m = max(max(s[i], s[i + 1]), m);
      m = largest<Lanes>(max(m, s[kHeld - 1]));
      if constexpr (Biased) {
        const float score = score_of(m);
        const bool follows = m != 0u && before - score <= 0x1p-21f * (1.0f + fabsf(score));
        near = near || (follows && j <= k);
        if (j >= k && !__ballot(follows)) break;
        full = j == (uint32_t)(Lanes * kSlots);
        if (full) break;
        before = score;
      }
      uint32_t at = 0xffffffffu;
#pragma unroll
      for (int i = kHeld - 1; i >= 0; --i) at = s[i] == m ? expert(i) : at;
      at = lowest<Lanes>(at);
      if (m == 0u) at = 0xffffffffu;
#pragma unroll
      for (int i = 0; i < kHeld; ++i) s[i] = at == expert(i) ? 0u : s[i];
      keep(j, at);
    }
    if constexpr (!Biased) return false;
    if (!__ballot(near)) return false;
    if (full) return near;
    double d[kSlots];
#pragma unroll
    for (int h = 0; h < kSlots; ++h) {
      d[h] = which[h] < 0 ? (double)kNever : score64(logit(which[h]), bias[which[h]]);
      rank[h] = which[h] < 0 ? rank[h] : 0u;
    }
#pragma unroll
    for (int h = 0; h < kSlots; ++h) {
      for (uint32_t l = 0; l < (uint32_t)Lanes && l + (uint32_t)(h * Lanes) < j; ++l) {
        const double o = __shfl(d[h], (int)l, Lanes);
        const int32_t ow = __shfl(which[h], (int)l, Lanes);
#pragma unroll
        for (int g = 0; g < kSlots; ++g) rank[g] += which[g] >= 0 && ow >= 0 && (o > d[g] || (o == d[g] && ow < which[g])) ? 1u : 0u;
      }
    }
    return false;
  }

  __device__ inline void rounds64(uint32_t k, const float* bias, const uint32_t (&s)[kHeld], bool again) {
    double d[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) d[i] = s[i] ? score64(logit((int32_t)expert(i)), bias[expert(i)]) : (double)kNever;
    for (uint32_t j = 0; j < k; ++j) {
      double best = (double)kNever;
      uint32_t at = 0xffffffffu;
#pragma unroll
      for (int i = 0; i < kHeld; ++i) {
        if (d[i] > best) {
          best = d[i];
          at = expert(i);
        }
      }
#pragma unroll
      for (int l = Lanes / 2; l > 0; l /= 2) {
        const double o = __shfl_xor(best, l);
        const uint32_t oa = (uint32_t)__shfl_xor((int)at, l);
        if (o > best || (o == best && oa < at)) {
          best = o;
          at = oa;
        }
      }
#pragma unroll
      for (int i = 0; i < kHeld; ++i) d[i] = at == expert(i) ? (double)kNever : d[i];
      if (again) keep(j, at);
    }
  }
};

// One token's experts and their weights; `marks`, where there is one, gets the token's bit for each expert chosen.
template <typename T, int Lanes, int Quads, bool Biased>
__device__ inline void choose(const RouteArgs& a, uint32_t t, uint32_t* marks, uint32_t words, uint32_t bit) {
  using C = Chooser<T, Lanes, Quads, Biased>;
  constexpr int kHeld = C::kHeld, kSlots = C::kSlots;
  C c;
  c.lane = threadIdx.x % Lanes;
  c.row = static_cast<const T*>(a.logits) + t * a.stride;
  float x[kHeld];
  uint32_t s[kHeld];
#pragma unroll
  for (int q = 0; q < Quads; ++q) {
    const uint32_t e = c.expert(4 * q);
    if (e + 4u <= a.n_experts) {
      const Four<T> f = *reinterpret_cast<const Four<T>*>(c.row + e);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * q + i] = (float)f.v[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * q + i] = e + (uint32_t)i < a.n_experts ? (float)c.row[e + i] : kNever;
    }
  }
#pragma unroll
  for (int q = 0; q < Quads; ++q) {
    Four<float> b{};
    if constexpr (Biased) {
      const uint32_t e = c.expert(4 * q);
      if (e + 4u <= a.n_experts) {
        b = *reinterpret_cast<const Four<float>*>(a.bias + e);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) b.v[i] = e + (uint32_t)i < a.n_experts ? a.bias[e + i] : 0.0f;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float& v = x[4 * q + i];
      v = C::tidy(v);
      float score = v;
      if constexpr (Biased) {
        score = sigmoid(v) + b.v[i];
        score = v > kNever && score == score ? score : kNever;
      }
      s[4 * q + i] = score > kNever ? key_of(score) : 0u;
    }
  }
  float sum = 1.0f, top = kNever;
  if (!a.sigmoid) {  // (the keys are the logits')
    uint32_t m = s[0];
#pragma unroll
    for (int i = 1; i < kHeld; ++i) m = max(m, s[i]);
    m = largest<Lanes>(m);
    top = m ? score_of(m) : kNever;
    if (!a.renorm) {  // (where the chosen are divided by their sum, that of all is no part of it)
      sum = 0.0f;
#pragma unroll
      for (int i = 0; i < kHeld; ++i) sum += x[i] > kNever ? exp_below(x[i] - top) : 0.0f;
      sum = in_all<Lanes>(sum);
    }
  }
#pragma unroll
  for (int h = 0; h < kSlots; ++h) {
    c.which[h] = -1;
    c.rank[h] = c.lane + (uint32_t)(h * Lanes);
  }
  if constexpr (Biased) {
    uint32_t once[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) once[i] = s[i];
    const bool again = c.rounds(a.k, a.bias, once);
    if (__ballot(again)) c.rounds64(a.k, a.bias, s, again);
  } else {
    c.rounds(a.k, nullptr, s);
  }
  float p[kSlots], l[kSlots], chosen = 0.0f, most = kNever, over = 0.0f;
#pragma unroll
  for (int h = 0; h < kSlots; ++h) {
    const bool is = c.which[h] >= 0 && c.rank[h] < a.k;
    l[h] = is ? c.logit(c.which[h]) : kNever;
    most = fmaxf(most, l[h]);
  }
  // Sigmoids that are divided by their sum are divided by exp(`over`) first, the chosen's largest logit where that is below 0: 64 bits would hold them,
  // 32 do not.  (Where 64 would not either, they are 0, so that a row of the type's lowest value has no weights.)
  if (a.sigmoid && a.renorm) over = fminf(join<Lanes>(most, [](float x, float y) { return fmaxf(x, y); }), 0.0f);
#pragma unroll
  for (int h = 0; h < kSlots; ++h) {
    p[h] = l[h] < (a.sigmoid ? kNoShare : -3.40282347e38f) ? 0.0f : a.sigmoid ? sigmoid_over(l[h], over) : exp_below(l[h] - top);
    chosen += p[h];
  }
  chosen = in_all<Lanes>(chosen);
  const float by = a.renorm ? chosen : sum;
#pragma unroll
  for (int h = 0; h < kSlots; ++h) {
    const uint32_t j = c.rank[h];
    if (j >= a.k) continue;
    a.expert[(uint64_t)t * a.k + j] = c.which[h];
    a.weight[(uint64_t)t * a.k + j] = c.which[h] < 0 || by == 0.0f ? 0.0f : p[h] / by * a.scale;
    if (marks && c.which[h] >= 0) atomicOr(&marks[(uint32_t)c.which[h] * words + bit / 32u], 1u << (bit & 31u));
  }
}

// Which tokens go to each expert is a bit each: an expert is chosen by a token once at most, so a token's rank among its
// expert's is the number of bits below its own.  `experts` holds bits [n_experts][words], first tokens `first` .. `first + tokens`.
__device__ inline void put_chosen(const RouteArgs& a, uint32_t first, uint32_t tokens, const uint32_t* bits, uint32_t words, const uint32_t* before) {
  for (uint32_t i = threadIdx.x; i < tokens * a.k; i += blockDim.x) {
    const int32_t e = a.expert[(uint64_t)first * a.k + i];
    const uint32_t t = i / a.k;
    int32_t to = -1;
    if (e >= 0) {
      const uint32_t* b = bits + (uint32_t)e * words;
      uint32_t rank = before[e] + (uint32_t)__builtin_popcount(b[t / 32u] & ((1u << (t & 31u)) - 1u));
      for (uint32_t w = 0; w < t / 32u; ++w) rank += (uint32_t)__builtin_popcount(b[w]);
      if (rank < a.n * a.k) {  // (counts that another replay wrote into the same workspace meanwhile are not followed out of token)
        to = (int32_t)rank;
        a.token[rank] = (int32_t)(first + t);
      }
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

__device__ inline void mark_chosen(const RouteArgs& a, uint32_t first, uint32_t tokens, uint32_t* bits, uint32_t words) {
  for (uint32_t i = threadIdx.x; i < tokens * a.k; i += blockDim.x) {
    const int32_t e = a.expert[(uint64_t)first * a.k + i];
    const uint32_t t = i / a.k;
    if (e >= 0) atomicOr(&bits[(uint32_t)e * words + t / 32u], 1u << (t & 31u));
  }
  lds_atomics_barrier();
}

// All tokens in order by one block of 1024, from their bits.  Shared memory: bits [n_experts][words], then before [n_experts].
__device__ inline void order_all(const RouteArgs& a, uint32_t* room, uint32_t words, uint32_t* meet) {
  uint32_t* before = room + a.n_experts * words;
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

// A handful of tokens: chosen and put in order by one block.
template <typename T, int Lanes, int Quads, bool Biased> __global__ void __launch_bounds__(1024) route_kernel(RouteArgs a) {
  extern __shared__ uint32_t room[];
  __shared__ uint32_t meet[16];
  const uint32_t words = (a.n + 31u) / 32u;
  for (uint32_t i = threadIdx.x; i < a.n_experts * words; i += 1024u) room[i] = 0u;
  __syncthreads();
  for (uint32_t t = threadIdx.x / Lanes; t < a.n; t += 1024u / Lanes) choose<T, Lanes, Quads, Biased>(a, t, room, words, t);
  lds_atomics_barrier();
  order_all(a, room, words, meet);
}

// Some more: put in order by one block when all are chosen.
__global__ void __launch_bounds__(1024) route_order_kernel(RouteArgs a) {
  extern __shared__ uint32_t room[];
  __shared__ uint32_t meet[16];
  const uint32_t words = (a.n + 31u) / 32u;
  for (uint32_t i = threadIdx.x; i < a.n_experts * words; i += 1024u) room[i] = 0u;
  __syncthreads();
  mark_chosen(a, 0u, a.n, room, words);
  order_all(a, room, words, meet);
}

// A chunk of tokens to a block of 1024 threads, and how many of them go to each expert; where that is not asked for, a block of any size chooses
// for as many as it can at once.
template <typename T, int Lanes, int Quads, bool Biased> __global__ void __launch_bounds__(1024) route_choose_kernel(RouteArgs a) {
  __shared__ uint32_t marks[2 * MAASO_EXPERT_MAX];
  if (!a.before) {
    const uint32_t t = (blockIdx.x * blockDim.x + threadIdx.x) / Lanes;
    if (t < a.n) choose<T, Lanes, Quads, Biased>(a, t, nullptr, 0u, 0u);
    return;
  }
  const uint32_t first = blockIdx.x * kChunk;
  for (uint32_t i = threadIdx.x; i < 2u * a.n_experts; i += 1024u) marks[i] = 0u;
  __syncthreads();
  for (uint32_t t = threadIdx.x / Lanes; t < kChunk && first + t < a.n; t += 1024u / Lanes) choose<T, Lanes, Quads, Biased>(a, first + t, marks, 2u, t);
  lds_atomics_barrier();
  for (uint32_t e = threadIdx.x; e < a.n_experts; e += 1024u)
    a.before[(uint64_t)blockIdx.x * a.n_experts + e] = (uint32_t)(__builtin_popcount(marks[2u * e]) + __builtin_popcount(marks[2u * e + 1u]));
}

// 16 experts to a block: their tokens before each chunk, and in all.  64 chunks side by side, the next 64 behind them.
__global__ void __launch_bounds__(1024) route_before_kernel(RouteArgs a) {
  __shared__ uint32_t sums[64][17];
  const uint32_t e = blockIdx.x * 16u + threadIdx.x % 16u, c = threadIdx.x / 16u;
  uint32_t seen = 0u;
  for (uint32_t base = 0; base < a.chunks; base += 64u) {
    const bool in = e < a.n_experts && base + c < a.chunks;
    uint32_t* p = a.before + (uint64_t)(base + c) * a.n_experts + e;
    const uint32_t mine = in ? *p : 0u;
    uint32_t upto = mine;  // over the chunks: neighbours are 16 lanes apart in a wave, and 4 rows of `sums` are a wave's
    uint32_t o = (uint32_t)__shfl_up((int)upto, 16);
    upto += (threadIdx.x & 63u) >= 16u ? o : 0u;
    o = (uint32_t)__shfl_up((int)upto, 32);
    upto += (threadIdx.x & 63u) >= 32u ? o : 0u;
    sums[c][threadIdx.x % 16u] = upto;
    __syncthreads();
    uint32_t below = 0u, all = 0u;
    for (uint32_t w = 0; w < 16u; ++w) {
      const uint32_t v = sums[4u * w + 3u][threadIdx.x % 16u];
      below += w < c / 4u ? v : 0u;
      all += v;
    }
    if (in) *p = seen + below + upto - mine;
    seen += all;
    __syncthreads();
  }
  if (c == 0u && e < a.n_experts) a.total[e] = seen;
}

__global__ void __launch_bounds__(1024) route_place_kernel(RouteArgs a) {
  __shared__ uint32_t marks[2 * MAASO_EXPERT_MAX], before[MAASO_EXPERT_MAX], meet[16];
  const uint32_t first = blockIdx.x * kChunk, tokens = min(kChunk, a.n - first), e = threadIdx.x;
  for (uint32_t i = threadIdx.x; i < 2u * a.n_experts; i += 1024u) marks[i] = 0u;
  uint32_t all;
  const uint32_t mine = e < a.n_experts ? a.total[e] : 0u, in_chunks = e < a.n_experts ? a.before[(uint64_t)blockIdx.x * a.n_experts + e] : 0u;
  const uint32_t at = block_before(mine, meet, all);  // (a barrier in it, behind the marks' zeros)
  if (e < a.n_experts) {
    before[e] = at + in_chunks;
    if (blockIdx.x == 0u) a.start[e] = (int32_t)at;
  }
  if (blockIdx.x == 0u && e == 0u) a.start[a.n_experts] = (int32_t)all;
  mark_chosen(a, first, tokens, marks, 2u);
  put_chosen(a, first, tokens, marks, 2u, before);
  for (uint32_t i = first * a.k + threadIdx.x; i < (first + tokens) * a.k; i += 1024u)
    if (i >= all) a.token[i] = -1;
}

}  // namespace maaso
