// Exponentials, and the gate of a feed-forward: silu(x) = x / (1 + exp(-x)).
#pragma once

#include <hip/hip_runtime.h>

namespace maaso {

// exp(d) for d <= 0 from the exponential to base 2; what the rounding of d log2(e) loses is made good in the first order.
__device__ inline float exp_below(float d) {
  constexpr float kLog2E = 1.44269504f, kRest = 1.92596299e-8f, kLn2 = 0.693147181f;  // log2(e) = kLog2E + kRest
  const float t = d * kLog2E;
  const float rest = fmaf(d, kRest, fmaf(d, kLog2E, -t));
  const float p = __builtin_amdgcn_exp2f(t);
  return t > -160.0f ? fmaf(p, rest * kLn2, p) : d != d ? d : 0.0f;
}

struct Halves {
  float e, r;  // exp(-|x|), which cannot overflow, and 1 / (1 + e), with one Newton step on the reciprocal
};
__device__ inline Halves halves(float x) {
  const float e = exp_below(-fabsf(x)), d = 1.0f + e, q = __builtin_amdgcn_rcpf(d);
  return {e, fmaf(q, fmaf(-d, q, 1.0f), q)};
}
__device__ inline float sigmoid(float x) {
  const Halves h = halves(x);
  return x < 0.0f ? h.e * h.r : h.r;
}
// sigmoid(x) / exp(s) for s <= 0, x <= s or s = 0: what shares of a sum can be taken of where sigmoid(x) itself is no number any more.
__device__ inline float sigmoid_over(float x, float s) {
  const float r = halves(x).r;
  return x < 0.0f ? exp_below(x - s) * r : r;
}
__device__ inline float silu(float x) { return x * sigmoid(x); }

}  // namespace maaso
