// Which kernel runs a dense product with 4-bit weights, and how it is cut (host).
#include <algorithm>
#include <cmath>

#include "linear4.h"

namespace aep {

// A tile's time for 4096 of K, of one that a CU has at a time or shares with others, by
// measurements with the weights in HBM (us; launch 3): 1 x 4096 x 4096 1x1 5.5, 1x2 6.1, 1x4
// 7.5; 1 x 14336 x 4096 1x1 12.7, 1x2 9.7, 1x4 9.1; 32 x 4096 x 4096 1x2 6.9, 1x4 8.0, 1x1 8.5, 2x2
// 8.9, 2x4 10.8; 32 x 14336 x 4096 2x4 12.4, 1x4 13.7, 2x2 14.9, 1x2 16.6; 64 x 4096 x 4096 1x4
// 7.8, 2x2 8.5, 1x2 9.3, 2x4 10.2; 128 x 4096 x 4096 2x4 9.8, 2x2 12.5, 4x4 14.5; 256 x 4096 x
// 4096 4x4 14.3, 2x4 14.6, 2x2 19.7; 128 x 14336 x 4096 2x4 26.4, 4x4 27.9, 2x2 33.2.  Eight
// waves; with four, or more steps in flight, all but the smallest tiles are slower.  8x8 is the tile
// kernel: 512 x 4096 x 4096 35, 4x4 29; 777 x 4096 x 4096 40, 4x4 55, 2x4 50; 1024 x 4096 x 4096
// 42, 4x4 65; 300 x 8000 x 1000 18, 2x4 27, 4x4 39.
RowsPlan rows4_plan(int m, int n, int k, bool tiles_128, int ncu) {
  struct Shape {
    int rf, cf;
    double us;
  };
  constexpr Shape kShapes[] = {{1, 1, 2.5}, {1, 2, 3.5}, {1, 4, 5.0}, {2, 2, 5.0}, {2, 4, 6.6}, {4, 4, 11.6}, {8, 8, 33.0}};
  RowsPlan best{0, 0, 1e300};
  for (const Shape& q : kShapes) {
    if (q.rf == 8 && !tiles_128) continue;
    const double tiles = (double)((m + q.rf * 16 - 1) / (q.rf * 16)) * ((n + q.cf * 16 - 1) / (q.cf * 16)) / ncu;
    // (of the largest tiles a CU holds one)
    const double rounds = tiles > 2.0 && q.rf < 4 ? tiles : std::ceil(tiles);
    const double us = 3.0 + rounds * (q.us * (double)k / 4096.0 + (q.rf == 8 ? 5.0 : 0.0));
    if (us < best.us) best = RowsPlan{q.rf, q.cf, us};
  }
  return best;
}

// Weights widened to bf16 first (their bytes at 4 TB/s and a launch), for the other tile kernel,
// where that is faster: 2048 x 4096 x 4096 76 us, in place 81; 777 x 4096 x 4096 54 and 40.
Linear4Plan linear4_plan(const LinearArgs& p, int nwg, int64_t max_bytes) {
  Linear4Plan r{};
  r.k8 = (p.k + 7) / 8 * 8;
  r.rows = rows4_plan(p.m, p.n, p.k, p.ldx < 1 << 22, nwg);
  if (p.n < 8 || p.k >= 1 << 22 || std::max(p.ldy, p.res ? p.ldr : 0) >= 1 << 22) return r;
  const double rows = r.rows.us;
  if (rows < 16.0) return r;  // less than any tiled product takes
  const int64_t w = (int64_t)p.n * r.k8 * 2;
  const int64_t x = !p.x_aligned || r.k8 != p.k || p.ldx >= 1 << 22 ? (int64_t)p.m * r.k8 * 2 : 0;
  if (w >= (int64_t)1 << 32 || x >= (int64_t)1 << 29 || w + x > max_bytes) return r;
  const LinearPlan& t = linear_plan(p.m, p.n, r.k8, false, p.wide, nwg, (max_bytes - w - x) / 4);
  if (t.us + 2.5 + (double)w * 1.27 / 4e6 + (x ? 2.5 + (double)x / 1.5e6 : 0.0) >= rows) return r;
  r.widen = true;
  r.w_bytes = w;
  r.x_bytes = x;
  r.tile_floats = t.cut.floats(p.n);
  return r;
}

}  // namespace aep
