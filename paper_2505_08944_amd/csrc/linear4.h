// The dense product with 4-bit weights: what its parts share.
#pragma once

#include "linear_tiles.h"

namespace aep {

constexpr int kLinear4Piece = 1088;  // bytes of 16 rows by 128 of K, packed (k_mx4.hip)
inline int linear4_steps(int k) { return (k + 127) / 128; }
inline int64_t linear4_pieces(int n, int k) { return (int64_t)((n + 15) / 16) * linear4_steps(k); }

hipError_t launch_mx4_quantize(const void* x, int x_dtype, int64_t ld, int64_t rows, int k, uint8_t* codes, uint8_t* scale,
                               hipStream_t s);
hipError_t launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scale, int64_t rows, int k, void* y, int y_dtype,
                                 int64_t ld, hipStream_t s);
hipError_t launch_linear4_pack(const uint8_t* codes, const uint8_t* scale, int n, int k, uint8_t* packed, hipStream_t s);
hipError_t launch_linear4_unpack(const uint8_t* packed, int n, int k, int k8, uint16_t* out, hipStream_t s);

// The tile of the kernels that take the codes as they are (k_linear4.hip; in 16s, 8 x 8: the tile
// kernel, if tiles_128), and its time in us.
RowsPlan rows4_plan(int m, int n, int k, bool tiles_128, int ncu);
hipError_t launch_linear4_rows(const LinearArgs& p, const RowsPlan& r, hipStream_t s);

// Whether the weights are widened to bf16 first, for the tile kernel, and the scratch
// of that: the weights, x where its rows are not 16-byte aligned, and the tiles' sums.
struct Linear4Plan {
  RowsPlan rows;  // (if not)
  bool widen;
  int k8;
  int64_t w_bytes, x_bytes, tile_floats;
  int64_t bytes() const { return w_bytes + x_bytes + tile_floats * 4; }
};
Linear4Plan linear4_plan(const LinearArgs& p, int nwg, int64_t max_bytes);
hipError_t launch_linear4(const LinearArgs& p, int nwg, void* scratch, int64_t bytes, hipStream_t s);

// Rows of k values of any alignment to rows of `bytes / rows` bytes, zeros behind (k_linear.hip).
hipError_t linear_align_bf16(const void* src, int64_t ld, int rows, int k, int64_t bytes, void* dst, hipStream_t s);

}  // namespace aep
