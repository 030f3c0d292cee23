// Dense product with its epilogue: y = f(s * (x W^T) + b) + r.
//
// Row kernel (this file's linear_rows_kernel): output tiles of up to 64 x 64,
// the waves of a workgroup split K and add their sums in LDS, in wave order.
// Operands go from global memory straight into MFMA fragments: what this
// kernel is for is bound by one operand's stream from HBM (few rows, or few
// channels), which every value leaves once, so LDS would only add a stop.
#include <limits.h>

#include <algorithm>

#include "linear_epilogue.h"
#include "linear_tiles.h"

namespace aep {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------- row kernel
// Element types of the operands: what one lane holds of a chunk of K, and how.
// bf16 / fp8: a chunk is 64 values of k; lane quarter h = lane / 16 holds k =
// 16 h .. 16 h + 15 of its row, in both operands alike, so MFMA step s pairs k
// = 16 h + 8 s + j of both.  f32: 32 values, k = 8 h .. 8 h + 7, eight steps
// of 16x16x4.
// N values of T from p on: 16-byte loads where the rows are aligned, else
// unaligned ones; values from `left` on are zeros.
template <typename T, int N, bool ALIGNED>
__device__ __forceinline__ void load_row(uint4* __restrict__ out, const T* __restrict__ p, int left, bool whole) {
  constexpr int PER = 16 / (int)sizeof(T);  // values per 16 bytes
  constexpr int Q = N / PER;
  if (whole) {
#pragma unroll
    for (int i = 0; i < Q; ++i) {
      if constexpr (ALIGNED)
        out[i] = *reinterpret_cast<const uint4*>(p + i * PER);
      else
        __builtin_memcpy(&out[i], p + i * PER, 16);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < Q; ++i) {
    if constexpr (ALIGNED) {  // 16 bytes end where the row does
      out[i] = make_uint4(0, 0, 0, 0);
      if (i * PER < left) out[i] = *reinterpret_cast<const uint4*>(p + i * PER);
    } else {
      T v[PER];
#pragma unroll
      for (int j = 0; j < PER; ++j) v[j] = i * PER + j < left ? p[i * PER + j] : T(0);
      __builtin_memcpy(&out[i], v, 16);
    }
  }
}

// XT / WT: storage types (uint16_t bf16, uint8_t e4m3, float).  RF x CF
// fragments of 16 x 16 outputs per workgroup.
template <typename XT, typename WT, int RF, int CF, int WAVES, bool ALIGNED>
__global__ __launch_bounds__(WAVES * 64) void linear_rows_kernel(const LinearArgs p) {
  constexpr bool F32 = sizeof(XT) == 4;
  constexpr int KC = F32 ? 32 : 64;      // k per chunk
  constexpr int LK = KC / 4;             // k per lane and chunk
  constexpr int XQ = LK * (int)sizeof(XT) / 16, WQ = LK * (int)sizeof(WT) / 16;
  constexpr int TM = RF * 16, TN = CF * 16, PITCH = TN + 4;
  __shared__ float part[WAVES][TM][PITCH];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rr = lane & 15, hh = lane >> 4;
  // an XCD gets a contiguous run of tiles, row tiles of a column band adjacent
  const int64_t per = gridDim.x >> 3;
  const int64_t tile = (int64_t)(blockIdx.x & 7) * per + (blockIdx.x >> 3);
  const int tm = (p.m + TM - 1) / TM;
  if (tile >= (int64_t)tm * ((p.n + TN - 1) / TN)) return;
  const int ti = (int)(tile % tm), tj = (int)(tile / tm);
  const int m0 = ti * TM, n0 = tj * TN;
  const int K = p.k, nch = (K + KC - 1) / KC;

  const XT* xr[RF];
  const WT* wr[CF];
#pragma unroll
  for (int i = 0; i < RF; ++i)
    xr[i] = reinterpret_cast<const XT*>(p.x) + (int64_t)min(m0 + i * 16 + rr, p.m - 1) * p.ldx + hh * LK;
#pragma unroll
  for (int j = 0; j < CF; ++j)
    wr[j] = reinterpret_cast<const WT*>(p.w) + (int64_t)min(n0 + j * 16 + rr, p.n - 1) * p.ldw + hh * LK;

  f32x4_t acc[RF][CF];
#pragma unroll
  for (int i = 0; i < RF; ++i)
#pragma unroll
    for (int j = 0; j < CF; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  uint4 xa[2][RF][XQ], wa[2][CF][WQ];
  auto load = [&](int b, int c) {
    const int k0 = c * KC, left = K - k0 - hh * LK;
    const bool whole = k0 + KC <= K;
#pragma unroll
    for (int j = 0; j < CF; ++j) load_row<WT, LK, ALIGNED>(wa[b][j], wr[j] + k0, left, whole);
#pragma unroll
    for (int i = 0; i < RF; ++i) load_row<XT, LK, ALIGNED>(xa[b][i], xr[i] + k0, left, whole);
  };
  auto mma = [&](int b) {
    if constexpr (F32) {
#pragma unroll
      for (int q = 0; q < XQ; ++q) {
#pragma unroll
        for (int i = 0; i < RF; ++i)
#pragma unroll
          for (int j = 0; j < CF; ++j) {
            const uint4 a = wa[b][j][q], v = xa[b][i][q];
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(v.x), acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(v.y), acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(v.z), acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(v.w), acc[i][j], 0, 0, 0);
          }
      }
    } else {
#pragma unroll
      for (int j = 0; j < CF; ++j) {
        bf16x8_t w[2];
        if constexpr (sizeof(WT) == 1) {
          const uint4 v = wa[b][j][0];
          const uint2 w0 = e4m3x4_to_bf16x4(v.x), w1 = e4m3x4_to_bf16x4(v.y);
          const uint2 w2 = e4m3x4_to_bf16x4(v.z), w3 = e4m3x4_to_bf16x4(v.w);
          w[0] = __builtin_bit_cast(bf16x8_t, make_uint4(w0.x, w0.y, w1.x, w1.y));
          w[1] = __builtin_bit_cast(bf16x8_t, make_uint4(w2.x, w2.y, w3.x, w3.y));
        } else {
          w[0] = __builtin_bit_cast(bf16x8_t, wa[b][j][0]);
          w[1] = __builtin_bit_cast(bf16x8_t, wa[b][j][1]);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < RF; ++i)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[s], __builtin_bit_cast(bf16x8_t, xa[b][i][s]),
                                                                acc[i][j], 0, 0, 0);
      }
    }
  };

  int c = wave;
  if (c < nch) {
    load(0, c);
    for (;;) {
      if (c + WAVES < nch) load(1, c + WAVES);
      mma(0);
      if ((c += WAVES) >= nch) break;
      if (c + WAVES < nch) load(0, c + WAVES);
      mma(1);
      if ((c += WAVES) >= nch) break;
    }
  }

  // lane: output row rr of a fragment, four consecutive columns 4 hh ..
#pragma unroll
  for (int i = 0; i < RF; ++i)
#pragma unroll
    for (int j = 0; j < CF; ++j)
      *reinterpret_cast<f32x4_t*>(&part[wave][i * 16 + rr][j * 16 + hh * 4]) = acc[i][j];
  __syncthreads();
  for (int e = tid; e < TM * (TN / 4); e += WAVES * 64) {
    const int r = e / (TN / 4), q = (e % (TN / 4)) * 4;
    if (m0 + r >= p.m || n0 + q >= p.n) continue;
    float4 s = *reinterpret_cast<const float4*>(&part[0][r][q]);
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
      const float4 v = *reinterpret_cast<const float4*>(&part[w][r][q]);
      s = make_float4(s.x + v.x, s.y + v.y, s.z + v.z, s.w + v.w);
    }
    linear_out4(p, m0 + r, n0 + q, p.n - n0 - q, s);
  }
}

template <typename XT, typename WT, int RF, int CF, bool ALIGNED>
static hipError_t rows_launch(const LinearArgs& p, hipStream_t s) {
  const int64_t tiles = (int64_t)((p.m + RF * 16 - 1) / (RF * 16)) * ((p.n + CF * 16 - 1) / (CF * 16));
  const int64_t grid = ((tiles + 7) / 8) * 8;
  if (grid > INT_MAX) return hipErrorInvalidValue;
  linear_rows_kernel<XT, WT, RF, CF, 8, ALIGNED><<<(unsigned)grid, 512, 0, s>>>(p);
  return hipGetLastError();
}

template <typename XT, typename WT, bool ALIGNED>
static hipError_t rows_tile(const LinearArgs& p, hipStream_t s) {
  if (p.m <= 16) return rows_launch<XT, WT, 1, 1, ALIGNED>(p, s);
  if (p.m <= 32) return rows_launch<XT, WT, 2, 1, ALIGNED>(p, s);
  if (p.n <= 64) return rows_launch<XT, WT, 2, 4, ALIGNED>(p, s);
  return rows_launch<XT, WT, 4, 2, ALIGNED>(p, s);
}

template <typename XT, typename WT>
static hipError_t rows_align(const LinearArgs& p, hipStream_t s) {
  const bool aligned = p.aligned;
  return aligned ? rows_tile<XT, WT, true>(p, s) : rows_tile<XT, WT, false>(p, s);
}

// Tiles need aligned rows, and offsets within a tile that fit 32 bits.
bool linear_uses_tiles(const LinearArgs& p) {
  if (p.w_dtype == kF32 || !p.aligned) return false;
  if (std::max(p.ldx, p.ldw) > (1 << 22)) return false;
  return p.m > 64 && p.n > 64;
}

hipError_t launch_linear(const LinearArgs& p, int nwg, float* scratch, int64_t scratch_floats, hipStream_t s) {
  if (linear_uses_tiles(p))
    return launch_linear_tiles(p, linear_cut(p.m, p.n, p.k, p.w_dtype == kFP8, nwg, scratch_floats), nwg, scratch, s);
  if (p.w_dtype == kF32) return rows_align<float, float>(p, s);
  if (p.w_dtype == kBF16) return rows_align<uint16_t, uint16_t>(p, s);
  return rows_align<uint16_t, uint8_t>(p, s);
}

}  // namespace aep
