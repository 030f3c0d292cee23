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

// e^-(a + lost) as m 2^n with m in [2^-1/2, 2^1/2], for a from 0 to 1000 and a lost that is
// small beside it: m is off by 2^-23 of its value, as the exponent's whole part leaves
// exactly (rounded as one f32, the exponent would put e^-80 off by 2^-17).
__device__ __forceinline__ float exp_parts(float a, float lost, int& n) {
#pragma clang fp contract(off)
  constexpr double kLog2E = 1.4426950408889634;
  constexpr float L = (float)kLog2E, L_lost = (float)(kLog2E - (double)L);
  const float whole = __builtin_rintf(a * L);
  n = -(int)whole;
  float f = __builtin_fmaf(a, L, -whole);
  f = __builtin_fmaf(a, L_lost, f);
  return __builtin_amdgcn_exp2f(-__builtin_fmaf(lost, L, f));
}
// v / (1 + e^-u) for u = +-(a + lost) of v's sign: as v e^u / (1 + e^u) below 0, so that
// nothing overflows.
__device__ __forceinline__ float gate(float v, float a, float lost) {
#pragma clang fp contract(off)
  int n;
  const float m = exp_parts(a, lost, n), e = __builtin_ldexpf(m, n);
  return v * (v < 0.f ? e : 1.f) * __builtin_amdgcn_rcpf(1.f + e);
}

// The activation for f32 results, and wherever there are few values: off by at most
// 2^-21 of its value (exponential and reciprocal 2^-23, 1 + e^u and the products 2^-24
// each), GELU by 2^-20, and by 2^-142, as e^u has steps of 2^-149 at least.  Products are
// not fused with what is added to them, here or to the result, so that equal values
// have equal results wherever they lie.  GELU is v Phi(v) with Phi(-a) = e^(-a^2 / 2) R(a)
// / 2, R(a) = erfcx(a / sqrt 2) a polynomial in 1 / (1 + 0.27 a) fitted to 2^-25 of
// its value for a up to 20 (in f32: 2^-21.3).  Arguments are cut off where the
// result is 0 or v.
template <int FN>
__device__ __forceinline__ float linear_fn(float v) {
#pragma clang fp contract(off)
  if constexpr (FN == kFnNone) return v;
  if constexpr (FN == kFnRelu) return v > 0.f ? v : v == v ? 0.f : v;  // NaN stays NaN
  if constexpr (FN == kFnSilu) return gate(v, fminf(fabsf(v), 360.f), 0.f);
  if constexpr (FN == kFnGeluTanh) {  // 1 + tanh u = 2 / (1 + e^-2u)
    const double a = fminf(fabsf(v), 20.f), u = 2.0 * 0.79788456080286536 * a * (1.0 + 0.044715 * a * a);
    const float hi = (float)u;
    return gate(v, hi, (float)(u - (double)hi));
  }
  constexpr float c[] = {0.215443328f, 0.215052918f, 0.203844741f, 0.143263772f, 0.217531502f, -0.141038328f, 0.341777891f,
                         -0.254003763f, 0.0581279807f};
  const float a = fminf(fabsf(v), 40.f), s = 0.5f * a * a;
  int n;
  const float m = exp_parts(s, __builtin_fmaf(0.5f * a, a, -s), n);
  const float z = __builtin_amdgcn_rcpf(1.f + 0.27f * a);
  float r = c[8];
#pragma unroll
  for (int i = 7; i >= 0; --i) r = __builtin_fmaf(r, z, c[i]);
  const float half = 0.5f * (r * z) * m;  // Phi(-|v|) = half 2^n
  const float tail = __builtin_ldexpf(half, n);
  return v * (v > 0.f ? 1.f - tail : tail);
}
__device__ __forceinline__ float linear_fn(int fn, float v) {
  switch (fn) {
    case kFnRelu: return linear_fn<kFnRelu>(v);
    case kFnSilu: return linear_fn<kFnSilu>(v);
    case kFnGelu: return linear_fn<kFnGelu>(v);
    case kFnGeluTanh: return linear_fn<kFnGeluTanh>(v);
    default: return v;
  }
}

// The activation for bf16 results of whole tiles, short enough to be laid out for every value of
// one: SILU and GELU_TANH as v / (1 + e^-u), with the hardware's exponential and
// reciprocal and u in f32: off by |u| 2^-22 of its value and a few steps of 2^-23 (below
// 2^-15 where the result is not lost: below u = -87 it is, of a size of 2^-119), where
// bf16's half step is 2^-9 .. 2^-8.  GELU with erf from Abramowitz and Stegun 7.1.26,
// whose error is at most 1.5e-7, here half of it times |v|.
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
