// The host side of the dense product's plan, built for the tests: linear_cut.hip
// with an empty HIP header.
#define __host__
#define __device__
typedef int hipError_t;
typedef void* hipStream_t;
#include <stddef.h>

#include "linear_cut.hip"

using namespace aep;

// out: tiles (1) or rows (0); then whole, rest, halves, p0, fam, pr, lrow, items, nrow, ncol; rf, cf
extern "C" void plan(int m, int n, int k, int fp8, int wide, int nwg, long long max_floats, int* out, double* us) {
  LinearArgs p{};
  p.m = m;
  p.n = n;
  p.k = k;
  p.w_dtype = fp8 ? kFP8 : kBF16;
  p.x_dtype = kBF16;
  p.ldx = p.ldw = k;
  p.ldy = p.ldr = n;
  p.x_aligned = p.w_aligned = 1;
  p.aligned = k % (fp8 ? 16 : 8) == 0;
  p.wide = wide;
  const TilesPlan t = linear_tiles_plan(p, nwg, max_floats);
  const LinearPlan& any = linear_plan(m, n, k, fp8, wide, nwg, max_floats);
  const LinearCut& c = any.cut;
  const RowsPlan r = rows_plan(m, n, k, 2, fp8 ? 1 : 2, nwg);
  const int v[] = {t.use, c.whole, c.rest, c.halves, c.p0, c.fam, c.pr, c.lrow, c.items, c.nrow, c.ncol, r.rf, r.cf};
  for (int i = 0; i < 13; ++i) out[i] = v[i];
  us[0] = any.us;
  us[1] = r.us;
  us[2] = (double)c.floats(n);
}
