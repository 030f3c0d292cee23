// The host side of the plan of the attention over a cache in 4 bits, built for the tests.
#include <stdint.h>

#include <algorithm>
#include <climits>

#include "attend4_plan.h"

using namespace aep;

// out: passes, then nc, workers, over, most of each; bytes of scratch
extern "C" long long plan(int batch, int total, int rows, int max_rows, int heads, int group, int d, long long max_len, int ncu,
                          int* out) {
  const Attend4Plan p = attend4_plan(batch, total, rows != 0, max_rows, heads, group, d, max_len, ncu);
  out[0] = p.passes;
  for (int i = 0; i < p.passes; ++i) {
    out[1 + 4 * i] = p.pass[i].nc;
    out[2 + 4 * i] = p.pass[i].workers;
    out[3 + 4 * i] = p.pass[i].over;
    out[4 + 4 * i] = p.pass[i].most;
  }
  return p.bytes;
}
