// Matrices to 4 bits and back (mx4.h), and the layout of 4-bit weights that the
// dense product reads.  All of it is bound by HBM: 14336 x 4096 from bf16 25 us (148 MB, 6 TB/s,
// part of it in the Infinity Cache), back 23, its layout for the product 14.
#include <algorithm>

#include "linear4.h"
#include "linear_epilogue.h"
#include "mx4.h"

namespace aep {

// Eight values of a row from p on, of which n exist (zeros behind), as f32.
template <typename T>
__device__ __forceinline__ void load8(const T* __restrict__ p, int n, float* v) {
  constexpr bool F32 = sizeof(T) == 4;
  if (n >= 8) {
    if constexpr (F32) {
      __builtin_memcpy(v, p, 32);
    } else {
      uint32_t w[4];
      __builtin_memcpy(w, p, 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf16_lo(w[i]);
        v[2 * i + 1] = bf16_hi(w[i]);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? (F32 ? (float)p[i] : bf16_lo((uint32_t)p[i])) : 0.f;
  }
}

// The first `n` bytes of a word, at any address.
__device__ __forceinline__ void store_bytes(uint8_t* p, uint32_t w, int n) {
  if (n >= 4) {
    __builtin_memcpy(p, &w, 4);
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < n) p[i] = (uint8_t)(w >> (8 * i));
  }
}

// Thread i of a row has its values 8 i .. 8 i + 7; the four threads of a quad share a
// block.  A workgroup takes 256 such runs of the matrix, row behind row.
template <typename T, bool BIG>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const T* __restrict__ x, int64_t ld, int64_t rows, int k, int runs,
                                                           uint8_t* __restrict__ codes, uint8_t* __restrict__ scale) {
  const int64_t i = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
  int64_t row;
  if constexpr (BIG)
    row = i / runs;
  else
    row = (uint32_t)i / (uint32_t)runs;
  if (row >= rows) return;  // (whole quads: runs is a multiple of 4)
  const int q = (int)(i - row * runs), at = q * 8;
  float v[8];
  load8(x + row * ld + at, k - at, v);
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[j]) & 0x7fffffffu);
  const uint32_t s = mx4_scale_byte(quad_max(m));
  const int64_t row_bytes = (k + 1) / 2;
  store_bytes(codes + row * row_bytes + at / 2, mx4_codes(v, mx4_scale(s == kMx4NaN ? 127 : s)), (k - at + 1) >> 1);
  if ((q & 3) == 0) scale[row * ((k + 31) / 32) + (q >> 2)] = (uint8_t)s;
}

template <bool F32, bool BIG>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint8_t* __restrict__ codes,
                                                             const uint8_t* __restrict__ scale, int64_t rows, int k, int runs,
                                                             void* __restrict__ y, int64_t ld) {
  const int64_t i = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
  int64_t row;
  if constexpr (BIG)
    row = i / runs;
  else
    row = (uint32_t)i / (uint32_t)runs;
  if (row >= rows) return;
  const int q = (int)(i - row * runs), at = q * 8, left = k - at;
  if (left <= 0) return;
  const uint8_t* p = codes + row * ((k + 1) / 2) + at / 2;
  uint32_t w = 0;
  if (left >= 7) {
    __builtin_memcpy(&w, p, 4);
  } else {
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (2 * j < left) w |= (uint32_t)p[j] << (8 * j);
  }
  const uint4 b = mx4_bf16x8(w, mx4_scale(scale[row * ((k + 31) / 32) + (q >> 2)]));
  const uint32_t v[4] = {b.x, b.y, b.z, b.w};
  if constexpr (F32) {
    float* o = reinterpret_cast<float*>(y) + row * ld + at;
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = j & 1 ? bf16_hi(v[j >> 1]) : bf16_lo(v[j >> 1]);
    if (left >= 8) {
      __builtin_memcpy(o, f, 32);
    } else {
#pragma unroll
      for (int j = 0; j < 7; ++j)
        if (j < left) o[j] = f[j];
    }
  } else {
    uint16_t* o = reinterpret_cast<uint16_t*>(y) + row * ld + at;
    if (left >= 8) {
      __builtin_memcpy(o, v, 16);
    } else {
#pragma unroll
      for (int j = 0; j < 7; ++j)
        if (j < left) o[j] = (uint16_t)(v[j >> 1] >> (16 * (j & 1)));
    }
  }
}

static dim3 grid_of(int64_t threads) {
  const int64_t blocks = (threads + 255) / 256, gx = std::min<int64_t>(blocks, 1 << 22);
  return dim3((unsigned)gx, (unsigned)((blocks + gx - 1) / gx));
}

hipError_t launch_mx4_quantize(const void* x, int x_dtype, int64_t ld, int64_t rows, int k, uint8_t* codes, uint8_t* scale,
                               hipStream_t s) {
  const int runs = (k + 31) / 32 * 4;
  const dim3 g = grid_of(rows * runs);
  const bool big = rows * runs + 256 >= (int64_t)1 << 32;
  const auto* xf = reinterpret_cast<const float*>(x);
  const auto* xb = reinterpret_cast<const uint16_t*>(x);
  if (x_dtype == kF32 && big) mx4_quantize_kernel<float, true><<<g, 256, 0, s>>>(xf, ld, rows, k, runs, codes, scale);
  if (x_dtype == kF32 && !big) mx4_quantize_kernel<float, false><<<g, 256, 0, s>>>(xf, ld, rows, k, runs, codes, scale);
  if (x_dtype == kBF16 && big) mx4_quantize_kernel<uint16_t, true><<<g, 256, 0, s>>>(xb, ld, rows, k, runs, codes, scale);
  if (x_dtype == kBF16 && !big) mx4_quantize_kernel<uint16_t, false><<<g, 256, 0, s>>>(xb, ld, rows, k, runs, codes, scale);
  return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scale, int64_t rows, int k, void* y, int y_dtype,
                                 int64_t ld, hipStream_t s) {
  const int runs = (k + 31) / 32 * 4;
  const dim3 g = grid_of(rows * runs);
  const bool big = rows * runs + 256 >= (int64_t)1 << 32;
  if (y_dtype == kF32 && big) mx4_dequantize_kernel<true, true><<<g, 256, 0, s>>>(codes, scale, rows, k, runs, y, ld);
  if (y_dtype == kF32 && !big) mx4_dequantize_kernel<true, false><<<g, 256, 0, s>>>(codes, scale, rows, k, runs, y, ld);
  if (y_dtype == kBF16 && big) mx4_dequantize_kernel<false, true><<<g, 256, 0, s>>>(codes, scale, rows, k, runs, y, ld);
  if (y_dtype == kBF16 && !big) mx4_dequantize_kernel<false, false><<<g, 256, 0, s>>>(codes, scale, rows, k, runs, y, ld);
  return hipGetLastError();
}

// ------------------------------------------------- weights of the dense product
// Packed: for each 16 rows and 128 of K a piece of 1088 bytes, K ascending within the
// rows: 64 lanes' 16 bytes (lane l: row l % 16, the block of 32 number l / 16), then
// their 64 scales.  What the matrix lacks of whole pieces is 0 with scale 2^0.

// One thread per block of 32: a wave makes a piece.
__global__ __launch_bounds__(256) void linear4_pack_kernel(const uint8_t* __restrict__ codes,
                                                           const uint8_t* __restrict__ scale, int n, int k, int steps,
                                                           int64_t pieces, uint8_t* __restrict__ out) {
  const int64_t piece = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (piece >= pieces) return;
  const int lane = threadIdx.x & 63;
  const int64_t row = piece / steps * 16 + (lane & 15);
  const int block = (int)(piece % steps) * 4 + (lane >> 4), left = k - block * 32;
  uint32_t w[4] = {0, 0, 0, 0};
  uint32_t s = 127;
  if (row < n && left > 0) {
    const uint8_t* p = codes + row * ((k + 1) / 2) + block * 16;
    if (left >= 32) {
      __builtin_memcpy(w, p, 16);
    } else {
      for (int j = 0; j < 16; ++j) {
        const int have = left - 2 * j;  // values from this byte on
        if (have > 0) w[j >> 2] |= (have > 1 ? (uint32_t)p[j] : (uint32_t)p[j] & 15u) << (8 * (j & 3));
      }
    }
    s = scale[row * ((k + 31) / 32) + block];
  }
  uint8_t* o = out + piece * kLinear4Piece;
  *reinterpret_cast<uint4*>(o + lane * 16) = make_uint4(w[0], w[1], w[2], w[3]);
  o[1024 + lane] = (uint8_t)s;
}

// Back to bf16 rows of k8 values (a multiple of 8, at most 128 times `steps`).
__global__ __launch_bounds__(256) void linear4_unpack_kernel(const uint8_t* __restrict__ packed, int n, int k8, int steps,
                                                             int64_t pieces, uint16_t* __restrict__ out) {
  const int64_t piece = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (piece >= pieces) return;
  const int lane = threadIdx.x & 63;
  const uint8_t* p = packed + piece * kLinear4Piece;
  // (16 lanes store 256 consecutive bytes of a row: lane l has the 8 values from 8 (l % 16) on of row 4 i + l / 16)
  const int row0 = (int)(piece / steps) * 16, k0 = (int)(piece % steps) * 128;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = i * 4 + (lane >> 4), q = lane & 15;  // row, 8 values of 128
    const int src = (q >> 2) * 16 + r;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(p + src * 16 + (q & 3) * 4);
    const uint4 v = mx4_bf16x8(w, mx4_scale(p[1024 + src]));
    const int row = row0 + r, at = k0 + q * 8;
    if (row < n && at < k8) *reinterpret_cast<uint4*>(out + (int64_t)row * k8 + at) = v;
  }
}

static dim3 piece_grid(int64_t pieces) { return grid_of(pieces * 64); }

hipError_t launch_linear4_pack(const uint8_t* codes, const uint8_t* scale, int n, int k, uint8_t* packed, hipStream_t s) {
  const int steps = linear4_steps(k);
  const int64_t pieces = linear4_pieces(n, k);
  linear4_pack_kernel<<<piece_grid(pieces), 256, 0, s>>>(codes, scale, n, k, steps, pieces, packed);
  return hipGetLastError();
}

hipError_t launch_linear4_unpack(const uint8_t* packed, int n, int k, int k8, uint16_t* out, hipStream_t s) {
  const int steps = linear4_steps(k);
  const int64_t pieces = linear4_pieces(n, k);
  linear4_unpack_kernel<<<piece_grid(pieces), 256, 0, s>>>(packed, n, k8, steps, pieces, out);
  return hipGetLastError();
}

}  // namespace aep
