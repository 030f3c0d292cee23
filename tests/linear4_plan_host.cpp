// The host side of the plan of a dense product with 4-bit weights, built for the tests:
// linear_cut.hip and linear4_cut.hip with an empty HIP header.
#define __host__
#define __device__
typedef int hipError_t;
typedef void* hipStream_t;
#include <stddef.h>

#include "linear_cut.hip"
#include "linear4_cut.hip"

using namespace aep;

// out: widened first (1) or not (0), rf, cf, k8; bytes of scratch
extern "C" long long plan4(int m, int n, int k, long long ldx, int aligned, long long max_bytes, int nwg, int* out) {
  LinearArgs p{};
  p.m = m;
  p.n = n;
  p.k = k;
  p.x_dtype = p.w_dtype = p.y_dtype = kBF16;
  p.ldx = ldx;
  p.ldy = p.ldr = n;
  p.x_aligned = aligned;
  p.wide = n % 8 == 0 ? kWideBf16 : 0;
  const Linear4Plan r = linear4_plan(p, nwg, max_bytes);
  out[0] = r.widen;
  out[1] = r.rows.rf;
  out[2] = r.rows.cf;
  out[3] = r.k8;
  return r.widen ? r.bytes() : 0;
}
