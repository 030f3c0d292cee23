// The epilogue of the dense product, shared by its kernels.
#pragma once

#include <type_traits>

#include "aep_device.h"
#include "aep_internal.h"

namespace aep {

// Four consecutive values of a bf16 or f32 row from `at` on, of which n exist.
// At once whatever their alignment: the load path takes unaligned addresses.
__device__ __forceinline__ float4 load4(const void* p, int dtype, int64_t at, int n) {
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (dtype == kF32) {
    const float* q = reinterpret_cast<const float*>(p) + at;
    if (n >= 4) {
      __builtin_memcpy(v, q, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < n) v[i] = q[i];
    }
  } else {
    const uint16_t* q = reinterpret_cast<const uint16_t*>(p) + at;
    if (n >= 4) {
      uint2 w;
      __builtin_memcpy(&w, q, 8);
      return make_float4(bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y));
    }
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < n) v[i] = bf16_lo(q[i]);
  }
  return make_float4(v[0], v[1], v[2], v[3]);
}

// f32 -> bf16, to nearest even; NaN stays NaN.
__device__ __forceinline__ uint32_t bf16_bits(float f) { return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  typedef __bf16 v2 __attribute__((ext_vector_type(2)));
  v2 v;
  v[0] = (__bf16)a;
  v[1] = (__bf16)b;
  return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ void store4(void* p, int dtype, int64_t at, int n, const float4 v) {
  const float a[4] = {v.x, v.y, v.z, v.w};
  if (dtype == kF32) {
    float* q = reinterpret_cast<float*>(p) + at;
    if (n >= 4) {
      __builtin_memcpy(q, a, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < n) q[i] = a[i];
    }
  } else {
    uint16_t* q = reinterpret_cast<uint16_t*>(p) + at;
    if (n >= 4) {
      const uint2 w = make_uint2(bf16_pair(a[0], a[1]), bf16_pair(a[2], a[3]));
      __builtin_memcpy(q, &w, 8);
    } else {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < n) q[i] = (uint16_t)bf16_bits(a[i]);
    }
  }
}

// v / (1 + e^-u) for f32 results: to within a few units of 2^-24.
__device__ __forceinline__ float gate(float v, float u) { return v / (1.f + expf(-u)); }

// The activation, accurate enough for an f32 result.  GELU through erfc, which
// keeps its relative accuracy where 1 + erf cancels; GELU_TANH as v / (1 +
// e^-2u), which does the same.
__device__ __forceinline__ float linear_fn(int fn, float v) {
  switch (fn) {
    case kFnRelu: return v > 0.f ? v : v == v ? 0.f : v;  // NaN stays NaN
    case kFnSilu: return gate(v, v);
    case kFnGelu: return 0.5f * v * erfcf(v * -0.70710678118654752f);
    case kFnGeluTanh: return gate(v, 2.f * 0.79788456080286536f * (v + 0.044715f * v * v * v));
    default: return v;
  }
}

// The activation for whole tiles, short enough to be laid out for every value of
// one: SILU and GELU_TANH as v / (1 + e^-u), with the hardware's exponential and
// reciprocal (2^-20 at |u| < 20; beyond, one of 1 and e^-u is lost); GELU with erf
// from Abramowitz and Stegun 7.1.26, whose error is at most 1.5e-7, here half of
// it times |v|.  Made for bf16 results (half a step: 2^-9 .. 2^-8 of them); an f32
// result keeps that relative error of 2^-20 (GELU: that absolute one, below what
// the sum's own roundings leave of v's size).
template <int FN>
__device__ __forceinline__ float linear_fn_tile(float v) {
  if constexpr (FN == kFnNone) return v;
  if constexpr (FN == kFnRelu) return v > 0.f ? v : v == v ? 0.f : v;
  if constexpr (FN == kFnSilu) return v * __builtin_amdgcn_rcpf(1.f + __expf(-v));
  if constexpr (FN == kFnGeluTanh) {
    constexpr float c0 = 2.f * 0.79788456f, c1 = 2.f * 0.79788456f * 0.044715f;
    return v * __builtin_amdgcn_rcpf(1.f + __expf(-v * (c0 + c1 * v * v)));
  }
  const float z = fabsf(v) * 0.70710678f;
  const float t = __builtin_amdgcn_rcpf(1.f + 0.3275911f * z);
  const float q = t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
  const float tail = 0.5f * q * __expf(-z * z);  // Phi(-|v|)
  return v * (v > 0.f ? 1.f - tail : tail);
}
// Calls f(activation) with the activation as a constant.
template <typename F>
__device__ __forceinline__ void by_fn(int fn, F f) {
  if (fn == kFnNone)
    f(std::integral_constant<int, kFnNone>{});
  else if (fn == kFnRelu)
    f(std::integral_constant<int, kFnRelu>{});
  else if (fn == kFnSilu)
    f(std::integral_constant<int, kFnSilu>{});
  else if (fn == kFnGelu)
    f(std::integral_constant<int, kFnGelu>{});
  else
    f(std::integral_constant<int, kFnGeluTanh>{});
}

// Four columns [c, c + 4) of row m: bias, activation, residual, one rounding.
// left: columns of the matrix from c on (may exceed 4).
__device__ __forceinline__ void linear_out4(const LinearArgs& p, int64_t m, int c, int left, float4 s) {
  const int64_t at = m * p.ldr + c;
  float4 b = make_float4(0.f, 0.f, 0.f, 0.f), r = b;
  if (p.scale) {
    const float4 q = load4(p.scale, kBF16, c, left);
    s = make_float4(s.x * q.x, s.y * q.y, s.z * q.z, s.w * q.w);
  }
  if (p.bias) b = load4(p.bias, p.bias_dtype, c, left);
  if (p.res) r = load4(p.res, p.res_dtype, at, left);
  s = make_float4(linear_fn(p.fn, s.x + b.x) + r.x, linear_fn(p.fn, s.y + b.y) + r.y, linear_fn(p.fn, s.z + b.z) + r.z,
                  linear_fn(p.fn, s.w + b.w) + r.w);
  store4(p.y, p.y_dtype, m * p.ldy + c, left, s);
}

}  // namespace aep
