// How a tiled dense product is cut (host).
#include <algorithm>

#include "linear_tiles.h"

namespace aep {

namespace {

constexpr int kMaxPieces = 8;
constexpr int kMinPieceSteps = 4;  // K steps of a piece
constexpr int64_t kMaxScratchFloats = (int64_t)24 << 20;

// us: a K step of a tile shape (256 x 256, 256 x 128, 128 x 128, 64 x 128), what
// an item takes besides, and the launch that adds the pieces' sums with its
// bytes.
struct Costs {
  double step[4], item[4], part[4], sums, sums_float;
};
constexpr Costs kBf16 = {{1.35, 0.85, 0.55, 0.45}, {6.0, 4.5, 4.0, 3.5}, {4.0, 2.5, 1.5, 1.0}, 4.0, 2.0e-6};
constexpr Costs kFp8 = {{1.50, 0.90, 0.60, 0.45}, {6.0, 4.5, 4.0, 3.5}, {4.0, 2.5, 1.5, 1.0}, 4.0, 2.0e-6};

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

LinearCut choose(int m, int n, int k, bool fp8, int nwg, int64_t max_floats) {
  const Costs& q = fp8 ? kFp8 : kBf16;
  const int KT = (k + 63) / 64;
  LinearCut c{};
  const int rem = m % 256;
  c.nrow = m / 256 + (rem > 128);
  c.fam = rem == 0 || rem > 128 ? 0 : rem > 64 ? 1 : 2;
  c.ncol = (n + 255) / 256;
  const int tiles = c.nrow * c.ncol;
  c.whole = tiles / nwg * nwg;
  c.rest = tiles - c.whole;
  LinearCut best{};
  double best_t = 1e300;
  const int last = c.last_tiles(n);
  const int max_p = std::max(1, std::min(kMaxPieces, KT / kMinPieceSteps));
  for (int halves = 1; halves <= 2; ++halves)
    for (int p0 = 1; p0 <= (c.rest ? max_p : 1); ++p0)
      for (int pr = 1; pr <= (c.fam ? max_p : 1); ++pr) {
        LinearCut t = c;
        t.halves = halves;
        t.p0 = p0;
        t.pr = pr;
        t.items = t.whole + t.rest_items() + last * pr;
        const int64_t fl = t.floats(n);
        if (fl > max_floats) continue;
        const int s0 = halves - 1, sr = 1 + t.fam;
        const double t0 = q.item[s0] + (double)KT / p0 * q.step[s0] + (p0 > 1 ? q.part[s0] : 0.0);
        const double tr = t.fam ? q.item[sr] + (double)KT / pr * q.step[sr] + (pr > 1 ? q.part[sr] : 0.0) : 0.0;
        double us = rounds_time(t.rest_items(), t0, (int64_t)last * pr, tr, nwg);
        if (fl) us += q.sums + q.sums_float * (double)fl;
        if (us < best_t) {
          best_t = us;
          best = t;
        }
      }
  return best;
}

}  // namespace

LinearCut linear_cut(int m, int n, int k, bool fp8, int nwg, int64_t max_floats) {
  // a few sizes come again and again: the last choices of this thread
  struct Seen {
    int m, n, k, fp8, nwg;
    int64_t max_floats;
    LinearCut cut;
  };
  static thread_local Seen seen[64];
  max_floats = std::min(max_floats, kMaxScratchFloats);
  const uint32_t h = ((uint32_t)m * 2654435761u ^ (uint32_t)n * 2246822519u ^ (uint32_t)k * 3266489917u) >> 26;
  Seen& s = seen[h];
  if (s.m != m || s.n != n || s.k != k || s.fp8 != (int)fp8 || s.nwg != nwg || s.max_floats != max_floats)
    s = Seen{m, n, k, (int)fp8, nwg, max_floats, choose(m, n, k, fp8, nwg, max_floats)};
  return s.cut;
}

}  // namespace aep
