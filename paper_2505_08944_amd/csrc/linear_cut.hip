// Which kernel runs a dense product, and how it is cut (host).
#include <algorithm>

#include "linear_tiles.h"

namespace aep {

namespace {

constexpr int kMaxPieces = 8;
constexpr int kMinPieceSteps = 4;  // K steps of a piece
constexpr int64_t kMaxScratchFloats = (int64_t)24 << 20;
constexpr int64_t kMaxCopiedBytes = (int64_t)512 << 20;  // of operands with unaligned rows

// us, fitted to launches of 65 .. 4096 rows with their operands in the Infinity
// Cache, each timed under all cuts worth trying (of 34 products, the chosen cut
// was more than 5% behind the best for two): a K step of a tile shape (256 x 256, 256 x 128, 128 x 128, 64 x 128), what
// an item takes besides, and the launch that adds the pieces' sums with its
// bytes.
// Results that do not go out as wide bf16 ones take an item longer (1024 of K, with
// bias, SiLU and residual in their type: 4096 x 4096 in tiles of 256 x 256 41 us, f32
// 56, others 66; 2048 x 2048 in 128 x 128 16.5, 20 and 22).
struct Costs {
  double step[4], item[4], part[4], sums, sums_float;
};
constexpr Costs kBf16 = {{1.25, 0.69, 0.47, 0.40}, {6.0, 5.4, 4.0, 3.6}, {4.0, 2.5, 1.5, 1.0}, 2.5, 1.0e-6};
constexpr double kResults[3][4] = {{16.0, 8.0, 4.0, 1.5}, {0.0, 0.0, 0.0, 0.0}, {6.0, 3.0, 2.0, 1.0}};  // by `wide`
constexpr Costs kFp8 = {{1.40, 0.70, 0.50, 0.43}, {6.0, 5.4, 4.0, 3.6}, {4.0, 2.5, 1.5, 1.0}, 2.5, 1.0e-6};

// The busiest workgroup's time in the rounds that hold a items of time ta and
// then b of time tb: these are dealt in turn, odd rounds in reverse, so a load
// changes along the workgroups only where a round passes from one kind to the
// other or ends.
double rounds_time(int64_t a, double ta, int64_t b, double tb, int nwg) {
  const int64_t n = a + b;
  const int64_t cand[] = {0, a % nwg, nwg - a % nwg, n % nwg, nwg - n % nwg, nwg - 1};
  double worst = 0.0;
  for (int64_t at0 : cand) {
    int64_t at = std::min<int64_t>(at0, nwg - 1);
    double sum = 0.0;
    for (int64_t base = 0; base < n; base += nwg) {
      const int64_t i = base + at;
      sum += i < a ? ta : i < n ? tb : 0.0;
      at = nwg - 1 - at;
    }
    worst = std::max(worst, sum);
  }
  return worst;
}

LinearPlan choose(int m, int n, int k, bool fp8, int wide, int nwg, int64_t max_floats) {
  const Costs& q = fp8 ? kFp8 : kBf16;
  const double* const result = kResults[wide];
  const int KT = (k + 63) / 64, rem = m % 256;
  const int max_p = std::max(1, std::min(kMaxPieces, KT / kMinPieceSteps));
  LinearPlan best{{}, 1e300};
  // rows: 256-row tiles and what is left; 128-row tiles; 64-row tiles
  for (int rows = 0; rows < 3; ++rows) {
    LinearCut c{};
    c.nrow = rows ? 0 : m / 256 + (rem > 128);
    c.fam = rows ? rows : rem == 0 || rem > 128 ? 0 : rem > 64 ? 1 : 2;
    c.lrow = rows ? (m + (256 >> rows) - 1) / (256 >> rows) : c.fam ? 1 : 0;
    c.ncol = (n + 255) / 256;
    const int64_t tiles = (int64_t)c.nrow * c.ncol, last = (int64_t)c.lrow * ((n + 127) / 128);
    if (rows && last > 4 * nwg) continue;  // many: larger tiles are better
    c.whole = (int)(tiles / nwg * nwg);
    c.rest = (int)(tiles - c.whole);
    for (int halves = 1; halves <= (c.rest ? 2 : 1); ++halves)
      for (int p0 = 1; p0 <= (c.rest ? max_p : 1); ++p0)
        for (int pr = 1; pr <= (c.fam ? max_p : 1); ++pr) {
          LinearCut t = c;
          t.halves = halves;
          t.p0 = p0;
          t.pr = pr;
          t.items = t.whole + t.rest_items() + (int)(last * pr);
          const int64_t fl = t.floats(n);
          if (fl > max_floats) continue;
          const int s0 = halves - 1, sr = 1 + t.fam;
          const double t0 = q.item[s0] + (double)KT / p0 * q.step[s0] + (p0 > 1 ? q.part[s0] : result[s0]);
          const double tr = t.fam ? q.item[sr] + (double)KT / pr * q.step[sr] + (pr > 1 ? q.part[sr] : result[sr]) : 0.0;
          double us = c.whole / nwg * (q.item[0] + KT * q.step[0] + result[0]) + rounds_time(t.rest_items(), t0, last * pr, tr, nwg);
          if (fl) us += q.sums + q.sums_float * (double)fl;
          if (us < best.us) best = LinearPlan{t, us};
        }
  }
  return best;
}

}  // namespace

const LinearPlan& linear_plan(int m, int n, int k, bool fp8, int wide, int nwg, int64_t max_floats) {
  // a few sizes come again and again: the last choices of this thread
  struct Seen {
    int m, n, k, fp8, wide, nwg;
    int64_t max_floats;
    LinearPlan plan;
  };
  static thread_local Seen seen[64];
  max_floats = std::min(max_floats, kMaxScratchFloats);
  const uint32_t h = ((uint32_t)m * 2654435761u ^ (uint32_t)n * 2246822519u ^ (uint32_t)k * 3266489917u) >> 26;
  Seen& s = seen[h];
  if (s.m != m || s.n != n || s.k != k || s.fp8 != (int)fp8 || s.wide != wide || s.nwg != nwg || s.max_floats != max_floats)
    s = Seen{m, n, k, (int)fp8, wide, nwg, max_floats, choose(m, n, k, fp8, wide, nwg, max_floats)};
  return s.plan;
}

// The tile with the least to load for the busiest CU: ceil(tiles / CUs) tiles of
// 16 (RF + CF) rows of K, at about 76 GB/s per CU, equal: the larger tile.  us
// of the choice and of the next best ones, operands in the Infinity Cache:
// 64 x 4096 x 4096 2x2 9.2, 1x4 10.5, 4x1 11.1, 4x2 12.6; 512 x 256 x 7168 1x2
// 12.0, 2x1 12.3, 2x2 13.5, 1x1 15.9; 128 x 4096 x 4096 2x4 12.9, 4x2 13.0, 2x2
// 14.9; 32 x 256 x 2048 1x1 4.6, 2x1 5.0, 2x2 5.4.
// f32: the same bytes at 120 GB/s and the MFMAs beside them, 0.9 us per fragment and
// 1024 of K (150 TFLOP/s on 256 CUs), 0.3 us per tile.  294 x 845 x 960 1x1 11.8, 2x1 13.2, 2x2
// 13.7, 2x4 (the choice by bytes alone) 14.2; 400 x 1500 x 1488 2x2 27.7, 2x1
// 31.2, 2x4 35.6; 512 x 2048 x 2048 2x2 48.1, 2x4 48.7, 1x1 63.3; 128 x 1024 x
// 1024 2x1 6.2, 1x1 6.3, 2x2 8.1, 2x4 13.0.
RowsPlan rows_plan(int m, int n, int k, int x_bytes, int w_bytes, int ncu) {
  constexpr int kShapes[][2] = {{2, 4}, {4, 2}, {2, 2}, {2, 1}, {1, 2}, {1, 1}};
  RowsPlan best{0, 0, 1e300};
  for (auto& q : kShapes) {
    const int rf = q[0], cf = q[1];
    const int64_t tiles = ((int64_t)(m + rf * 16 - 1) / (rf * 16)) * ((n + cf * 16 - 1) / (cf * 16));
    const double bytes = 16.0 * (rf * x_bytes + cf * w_bytes) * (double)k;
    const double tile = x_bytes == 4 ? 0.3 + bytes / 120e3 + 0.88e-3 * rf * cf * (double)k : bytes / 76e3;
    const double us = 3.0 + (double)((tiles + ncu - 1) / ncu) * tile;
    if (us < best.us) best = RowsPlan{rf, cf, us};
  }
  return best;
}

// Tiles where they are faster by both kernels' times (fitted to measurements
// of 48 .. 2048 rows, 64 .. 14336 columns and K = 1024 .. 14336: 384 x 4096 x
// 4096 rows 30, tiles 27 us; 256 x 4096 x 4096 22 and 25; 2048 x 1024 x 1024 15
// and 17; 96 x 14336 x 4096 32 and 29; 2048 x 4096 x 4096 160 and 47).  They need
// offsets within a tile that fit 31 bits.  With rows that have to be copied first:
// 777 x 2000 x 2001 rows 41, tiles 32; 1000 x 5000 x 2731 149 and 57; 2048 x 4096 x
// 4095 325 and 81, fp8 288 and 79; 4096 x 4096 x 1001 235 and 48.
TilesPlan linear_tiles_plan(const LinearArgs& p, int nwg, int64_t max_floats) {
  TilesPlan r{};
  if (p.w_dtype == kF32 || p.n < 8) return r;
  const int es = p.w_dtype == kFP8 ? 1 : 2, per = 16 / es;
  if (p.k >= 1 << 22 || std::max(p.ldy, p.res ? p.ldr : 0) >= 1 << 22) return r;
  r.k = (p.k + per - 1) / per * per;
  if (r.k != p.k || !p.x_aligned) r.x_bytes = (int64_t)p.m * r.k * 2;
  if (r.k != p.k || !p.w_aligned) r.w_bytes = (int64_t)p.n * r.k * es;
  if ((!r.x_bytes && p.ldx >= 1 << 22) || (!r.w_bytes && p.ldw >= 1 << 22)) return r;
  const int64_t copied = r.x_bytes + r.w_bytes;
  if (copied > kMaxCopiedBytes || copied / 4 > max_floats) return r;
  // (rows of any alignment take the row kernel half as long again)
  const double rows = rows_plan(p.m, p.n, p.k, 2, es, nwg).us * (p.aligned ? 1.0 : 1.5);
  if (rows < 16.0) return r;  // less than any tiled product takes
  const LinearPlan& t = linear_plan(p.m, p.n, r.k, es == 1, p.wide, nwg, max_floats - copied / 4);
  const double copies = (r.x_bytes ? 2.5 : 0.0) + (r.w_bytes ? 2.5 : 0.0) + (double)copied / 1.5e6;
  r.cut = t.cut;
  r.use = t.us + copies < rows;
  return r;
}

}  // namespace aep
