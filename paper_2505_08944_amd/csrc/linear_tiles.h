// Work division of the tiled dense product: shared by the host, which chooses
// the cut, the tile kernel and the kernel that adds the pieces' sums.
//
// Rows are covered by 256-row tiles (family 0) and, where 128 or fewer are
// left, by one row of tiles of 128 or 64 rows (family 1 or 2); or by rows of
// these alone.  Tiles of family 0 have 256 columns; full rounds of the grid of
// them are one item each.  What is left of them, a partial round, is cut into
// column halves or not, and these along K into pieces; tiles of the other
// families have 128 columns and are cut along K alone.  Pieces leave their f32
// sums in the scratch, one tile after another, where a second launch adds them
// in piece order.
#pragma once

#include "aep_internal.h"

namespace aep {

struct LinearCut {
  int nrow, ncol;   // 256 x 256 tiles: rows and columns of them
  int whole;        // tiles of family 0 that are one item each
  int rest;         // the others
  int halves;       // 2: these are cut into column halves, 1: not
  int p0;           // pieces along K of each of these
  int fam, pr;      // family of the last rows' tiles (0: none) and their pieces
  int lrow;         // rows of these tiles
  int items;        // all in all
  __host__ __device__ int rest_parts() const { return rest * halves; }         // tiles or halves
  __host__ __device__ int rest_items() const { return rest_parts() * p0; }
  __host__ __device__ int last_tiles(int n) const { return lrow * ((n + 127) / 128); }
  // f32 values of scratch; part q of a tile or half lies at its first float + q * its size
  __host__ __device__ int64_t rest_floats() const { return p0 > 1 ? (int64_t)rest_items() * (65536 / halves) : 0; }
  __host__ __device__ int64_t floats(int n) const {
    return rest_floats() + (pr > 1 ? (int64_t)last_tiles(n) * pr * (32768 >> fam) : 0);
  }
};

// The cheapest cut of a product of these sizes, its results going out as `wide`
// says, on nwg workgroups whose pieces' sums take at most max_floats of scratch,
// and its time.
struct LinearPlan {
  LinearCut cut;
  double us;
};
const LinearPlan& linear_plan(int m, int n, int k, bool fp8, int wide, int nwg, int64_t max_floats);
// The row kernel's tile (fragments of rows and columns) and its time.
struct RowsPlan {
  int rf, cf;
  double us;
};
RowsPlan rows_plan(int m, int n, int k, int x_bytes, int w_bytes, int ncu);
// Whether the tile kernel takes the product (or the row kernel), and then how.
// Operands whose rows are not 16-byte aligned are copied to rows of k values first,
// zeros behind their own, into the scratch behind the pieces' sums.
struct TilesPlan {
  bool use;
  LinearCut cut;
  int k;
  int64_t x_bytes, w_bytes;  // of the copies (0: none)
  int64_t bytes(int n) const { return cut.floats(n) * 4 + x_bytes + w_bytes; }
};
TilesPlan linear_tiles_plan(const LinearArgs& p, int nwg, int64_t max_floats);
hipError_t launch_linear_tiles(const LinearArgs& p, const LinearCut& c, int nwg, float* scratch, hipStream_t s);

}  // namespace aep
