// 16- and 8-bit floating types of the caches and of queries: loads, exact widenings, roundings to nearest even.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace maaso {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Before and after the stores of a branch that go past the caches: the compiler would make one of the two branches' stores,
// and forget which kind they are.
__device__ inline void keep_apart() { asm volatile("" ::: "memory"); }

struct E4m3 { uint8_t bits; };  // the 8-bit type of a cache, as a template's argument

template <typename T> struct Vec;
template <> struct Vec<__bf16> { using x2 = bf16x2; using x8 = bf16x8; };
template <> struct Vec<_Float16> { using x2 = f16x2; using x8 = f16x8; };

// Two values, each rounded to the nearest: one conversion instruction for either type.
template <typename T> __device__ inline typename Vec<T>::x2 narrow2(float a, float b) {
  return __builtin_convertvector((f32x2){a, b}, typename Vec<T>::x2);
}

template <typename T> __device__ inline typename Vec<T>::x8 narrow8(const float (&x)[8]) {
  typename Vec<T>::x8 r;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const auto v = narrow2<T>(x[2 * k], x[2 * k + 1]);
    r[2 * k] = v[0];
    r[2 * k + 1] = v[1];
  }
  return r;
}

// Eight 8-bit values to 16 bits: exact in both types (4 bits of mantissa, exponents -9 .. 8).
template <typename T> __device__ inline typename Vec<T>::x8 widen8(u32x2 b);
template <> __device__ inline bf16x8 widen8<__bf16>(u32x2 b) {
  bf16x8 r;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b[k], 1.0f, false);
    const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b[k], 1.0f, true);
    r[4 * k] = lo[0]; r[4 * k + 1] = lo[1]; r[4 * k + 2] = hi[0]; r[4 * k + 3] = hi[1];
  }
  return r;
}
template <> __device__ inline f16x8 widen8<_Float16>(u32x2 b) {
  f16x8 r;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const f16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b[k], 1.0f, false);
    const f16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b[k], 1.0f, true);
    r[4 * k] = lo[0]; r[4 * k + 1] = lo[1]; r[4 * k + 2] = hi[0]; r[4 * k + 3] = hi[1];
  }
  return r;
}

// To 8 bits: to the nearest, at most 448 in magnitude (an infinity too), NaN stays NaN.
__device__ inline float e4m3_range(float x) { return x != x ? x : fminf(fmaxf(x, -448.0f), 448.0f); }
__device__ inline uint32_t e4m3_pack4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(a), e4m3_range(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(c), e4m3_range(d), r, true);
}

__device__ inline f32x4 mfma_16x16x32(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x4 mfma_16x16x32(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 mfma_32x32x16(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 mfma_32x32x16(f16x8 a, f16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

}  // namespace maaso
