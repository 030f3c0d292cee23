// The activations of the dense product's epilogue, built for the tests on the
// host, whose exp2f, division and conversions stand in for the hardware's.
#include <math.h>
#include <stdint.h>
#include <string.h>
#define __device__
#define __host__
#define __forceinline__ inline
struct float4 {
  float x, y, z, w;
};
struct uint2 {
  unsigned x, y;
};
struct uint4 {
  unsigned x, y, z, w;
};
static inline float4 make_float4(float x, float y, float z, float w) { return {x, y, z, w}; }
static inline uint2 make_uint2(unsigned x, unsigned y) { return {x, y}; }
static inline float __uint_as_float(unsigned u) {
  float f;
  memcpy(&f, &u, 4);
  return f;
}
static inline unsigned __float_as_uint(float f) {
  unsigned u;
  memcpy(&u, &f, 4);
  return u;
}
typedef int hipError_t;
typedef void* hipStream_t;
#define __bf16 unsigned short
#define __expf expf
#define __builtin_amdgcn_rcpf(x) (1.f / (x))
#define __builtin_amdgcn_exp2f(x) exp2f(x)
#define __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, h) (bf16x2_t{})

#include "linear_epilogue.h"

using namespace aep;

// exact: the activation of f32 results and of rows; else that of whole bf16 tiles.
extern "C" void activations(int exact, int fn, const float* v, float* y, long n) {
  for (long i = 0; i < n; ++i) {
    if (exact)
      y[i] = linear_fn(fn, v[i]);
    else
      by_fn(fn, [&](auto f) { y[i] = linear_fn_tile<f()>(v[i]); });
  }
}
