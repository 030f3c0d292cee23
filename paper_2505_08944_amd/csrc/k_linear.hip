// Dense product with its epilogue: y = f(s * (x W^T) + b) + r.
//
// Row kernel (linear_rows_kernel): output tiles of up to 64 x 32, the waves of a
// workgroup split K and add their sums in LDS, in wave order.  It is for
// products that one operand's stream bounds (few rows, or few channels) and for
// f32; the tile kernel (k_linear_tiles.hip) takes the others (linear_cut.hip), rows
// of other alignments than 16 bytes through aligned copies.  Measured, us per call
// of a captured run of them, with the operands in the Infinity Cache and (in brackets)
// in HBM: 32 x 4096 x 4096 8.3 (11.3; its bytes at the rate of a large copy 6.6), 1 x
// 14336 x 4096 fp8 12.5 (16.7; 11.3), 8192 x 64 x 2048 9.0 (12.4; 6.9), an empty
// launch 1.5.
#include <algorithm>

#include "linear4.h"
#include "linear_epilogue.h"

namespace aep {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------- row kernel
// A chunk of K is 128 bytes of an x row (64 bf16 or 32 f32 values) and the
// same values of k of a W row.  A wave reads 16 rows by 64 bytes per load, the
// four lanes of a quad 64 consecutive bytes: lanes that read a row each, as an
// MFMA operand lies in them, take the load path 64 cycles per load, four times
// as long (32 x 4096 x 4096: 13.4 us).  The way from that order to the
// operand's is through the wave's own LDS, in order and without a barrier:
// lane l's 16 bytes go to place l; piece q of row r comes to lie at place 4 r +
// (q ^ (r / 4)), from where 16 lanes that read one piece of 16 rows hit all banks.

// 16 bytes of a row at p: unaligned ones where the rows are.
template <bool ALIGNED, typename T>
__device__ __forceinline__ uint4 load16(const T* __restrict__ p) {
  uint4 v;
  if constexpr (ALIGNED)
    v = *reinterpret_cast<const uint4*>(p);
  else
    __builtin_memcpy(&v, p, 16);
  return v;
}
// The same at the end of a row: values from `left` on are zeros.
template <bool ALIGNED, typename T>
__device__ __forceinline__ uint4 load16_end(const T* __restrict__ p, int left) {
  constexpr int PER = 16 / (int)sizeof(T);
  if constexpr (ALIGNED) {  // 16 bytes end where the row does
    return left > 0 ? *reinterpret_cast<const uint4*>(p) : make_uint4(0, 0, 0, 0);
  } else {
    T v[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) v[j] = j < left ? p[j] : T(0);
    uint4 o;
    __builtin_memcpy(&o, v, 16);
    return o;
  }
}

// XT / WT: storage types (uint16_t bf16, uint8_t e4m3, float).  RF x CF
// fragments of 16 x 16 outputs per workgroup, WAVES waves, which split K, each
// with D chunks of it in flight.
template <typename XT, typename WT, int RF, int CF, int WAVES, int D, bool ALIGNED>
__global__ __launch_bounds__(WAVES * 64) void linear_rows_kernel(const LinearArgs p) {
  constexpr bool F32 = sizeof(XT) == 4, FP8 = sizeof(WT) == 1;
  constexpr int KC = 128 / (int)sizeof(XT);  // k per chunk
  constexpr int XQ = 2, WQ = FP8 ? 1 : 2;    // loads per fragment and chunk
  constexpr int XP = 16 / (int)sizeof(XT), WP = 16 / (int)sizeof(WT);  // values per 16 bytes
  constexpr int TM = RF * 16, TN = CF * 16, PITCH = TN + 4;
  constexpr int kStage = (RF * XQ + CF * WQ) * 1024;  // a wave's chunk
  constexpr int kPart = TM * PITCH * 4;               // its sums
  __shared__ __attribute__((aligned(1024))) unsigned char smem[WAVES * (kStage > kPart ? kStage : kPart)];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rr = lane & 15, hh = lane >> 4;
  // an XCD gets a contiguous run of tiles, row tiles of a column band adjacent
  const int64_t per = gridDim.x >> 3;
  const int64_t tile = (int64_t)blockIdx.y * gridDim.x + (int64_t)(blockIdx.x & 7) * per + (blockIdx.x >> 3);
  const int tm = (p.m + TM - 1) / TM;
  if (tile >= (int64_t)tm * ((p.n + TN - 1) / TN)) return;
  const int ti = (int)(tile % tm), tj = (int)(tile / tm);
  const int m0 = ti * TM, n0 = tj * TN;
  const int K = p.k, nch = K / KC;  // whole chunks

  // this lane's row and 16-byte piece of a load
  const int lr = lane >> 2, lq = (lane & 3) ^ (lane >> 4);
  const XT* xr[RF];
  const WT* wr[CF];
#pragma unroll
  for (int i = 0; i < RF; ++i)
    xr[i] = reinterpret_cast<const XT*>(p.x) + (int64_t)min(m0 + i * 16 + lr, p.m - 1) * p.ldx + lq * XP;
#pragma unroll
  for (int j = 0; j < CF; ++j)
    wr[j] = reinterpret_cast<const WT*>(p.w) + (int64_t)min(n0 + j * 16 + lr, p.n - 1) * p.ldw + lq * WP;

  f32x4_t acc[RF][CF];
#pragma unroll
  for (int i = 0; i < RF; ++i)
#pragma unroll
    for (int j = 0; j < CF; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  uint4 xa[D][RF][XQ], wa[D][CF][WQ];
  auto load = [&](int b, int c) {
    const int k0 = c * KC;
#pragma unroll
    for (int j = 0; j < CF; ++j)
#pragma unroll
      for (int q = 0; q < WQ; ++q) wa[b][j][q] = load16<ALIGNED>(wr[j] + k0 + q * 4 * WP);
#pragma unroll
    for (int i = 0; i < RF; ++i)
#pragma unroll
      for (int q = 0; q < XQ; ++q) xa[b][i][q] = load16<ALIGNED>(xr[i] + k0 + q * 4 * XP);
  };
  unsigned char* mine = smem + wave * kStage;
  // 16 bytes of row rr of a fragment: piece q (of 8, or 4 for fp8 W)
  auto piece = [&](const unsigned char* frag, int q) {
    return *reinterpret_cast<const uint4*>(frag + (q >> 2) * 1024 + (rr * 4 + ((q & 3) ^ (rr >> 2))) * 16);
  };
  // One wave's LDS accesses are carried out in the order in which they were issued: the
  // compiler only has to keep it, across lanes that it does not know to share values.
  auto wave_order = [&] {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  auto mma = [&](int b) {
    wave_order();
    unsigned char* at = mine;
#pragma unroll
    for (int j = 0; j < CF; ++j)
#pragma unroll
      for (int q = 0; q < WQ; ++q, at += 1024) *reinterpret_cast<uint4*>(at + lane * 16) = wa[b][j][q];
#pragma unroll
    for (int i = 0; i < RF; ++i)
#pragma unroll
      for (int q = 0; q < XQ; ++q, at += 1024) *reinterpret_cast<uint4*>(at + lane * 16) = xa[b][i][q];
    wave_order();
    const unsigned char* xs = mine + CF * WQ * 1024;
    uint4 x[RF][2], w[CF][2];
#pragma unroll
    for (int j = 0; j < CF; ++j) {
      if constexpr (FP8) {
        const uint4 v = piece(mine + j * 1024, hh);  // k = 16 hh ..
        const uint2 w0 = e4m3x4_to_bf16x4(v.x), w1 = e4m3x4_to_bf16x4(v.y);
        const uint2 w2 = e4m3x4_to_bf16x4(v.z), w3 = e4m3x4_to_bf16x4(v.w);
        w[j][0] = make_uint4(w0.x, w0.y, w1.x, w1.y);
        w[j][1] = make_uint4(w2.x, w2.y, w3.x, w3.y);
      } else {
#pragma unroll
        for (int s = 0; s < 2; ++s) w[j][s] = piece(mine + j * 2048, 4 * s + hh);
      }
    }
#pragma unroll
    for (int i = 0; i < RF; ++i)
#pragma unroll
      for (int s = 0; s < 2; ++s) x[i][s] = piece(xs + i * 2048, FP8 ? 2 * hh + s : 4 * s + hh);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < RF; ++i)
#pragma unroll
        for (int j = 0; j < CF; ++j) {
          if constexpr (F32) {
            const uint4 a = w[j][s], v = x[i][s];
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(v.x), acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(v.y), acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(v.z), acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(v.w), acc[i][j], 0, 0, 0);
          } else {
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w[j][s]),
                                                                __builtin_bit_cast(bf16x8_t, x[i][s]), acc[i][j], 0, 0, 0);
          }
        }
  };

  // This wave's chunks, D at a time.  No branch stands between the loads of the
  // loop, so that the wait for one chunk leaves the later ones in flight.
  int c = wave, n = (nch - wave + WAVES - 1) / WAVES;
  if (n >= D) {
#pragma unroll
    for (int b = 0; b < D; ++b) load(b, c + b * WAVES);
    for (; n >= 2 * D; n -= D, c += D * WAVES) {
#pragma unroll
      for (int b = 0; b < D; ++b) {
        mma(b);
        load(b, c + (b + D) * WAVES);
      }
    }
#pragma unroll
    for (int b = 0; b < D; ++b) {
      mma(b);
      if (b < n - D) load(b, c + (b + D) * WAVES);
    }
    n -= D;
  } else {
#pragma unroll
    for (int b = 0; b < D - 1; ++b)
      if (b < n) load(b, c + b * WAVES);
  }
#pragma unroll
  for (int b = 0; b < D - 1; ++b)
    if (b < n) mma(b);
  if (K % KC && wave == nch % WAVES) {
    const int k0 = nch * KC;
#pragma unroll
    for (int j = 0; j < CF; ++j)
#pragma unroll
      for (int q = 0; q < WQ; ++q)
        wa[0][j][q] = load16_end<ALIGNED>(wr[j] + k0 + q * 4 * WP, K - k0 - (q * 4 + lq) * WP);
#pragma unroll
    for (int i = 0; i < RF; ++i)
#pragma unroll
      for (int q = 0; q < XQ; ++q)
        xa[0][i][q] = load16_end<ALIGNED>(xr[i] + k0 + q * 4 * XP, K - k0 - (q * 4 + lq) * XP);
    mma(0);
  }

  // lane: output row rr of a fragment, four consecutive columns 4 hh ..
  __syncthreads();  // the sums take the chunks' place
  float* part = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int i = 0; i < RF; ++i)
#pragma unroll
    for (int j = 0; j < CF; ++j)
      *reinterpret_cast<f32x4_t*>(part + (wave * TM + i * 16 + rr) * PITCH + j * 16 + hh * 4) = acc[i][j];
  __syncthreads();
  for (int e = tid; e < TM * (TN / 4); e += WAVES * 64) {
    const int r = e / (TN / 4), q = (e % (TN / 4)) * 4;
    if (m0 + r >= p.m || n0 + q >= p.n) continue;
    float4 s = *reinterpret_cast<const float4*>(part + r * PITCH + q);
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
      const float4 v = *reinterpret_cast<const float4*>(part + (w * TM + r) * PITCH + q);
      s = make_float4(s.x + v.x, s.y + v.y, s.z + v.z, s.w + v.w);
    }
    linear_out4(p, m0 + r, n0 + q, p.n - n0 - q, s);
  }
}

template <typename XT, typename WT, int RF, int CF, int WAVES, int D, bool ALIGNED>
static hipError_t rows_launch(const LinearArgs& p, hipStream_t s) {
  const int64_t tiles = (int64_t)((p.m + RF * 16 - 1) / (RF * 16)) * ((p.n + CF * 16 - 1) / (CF * 16));
  // (at most 2^30 tiles; a grid's side has fewer than 2^32 threads)
  const int64_t gx = std::min<int64_t>((tiles + 7) / 8 * 8, 1 << 22);
  const dim3 grid((unsigned)gx, (unsigned)((tiles + gx - 1) / gx));
  linear_rows_kernel<XT, WT, RF, CF, WAVES, D, ALIGNED><<<grid, WAVES * 64, 0, s>>>(p);
  return hipGetLastError();
}

// Waves and chunks in flight: 4 and 4 (2 where a chunk fills the registers), us
// against 8 waves for 32 x 4096 x 4096 7.9 and 8.7, 8192 x 64 x 2048 8.9 and 9.4;
// one fragment is for few tiles, whose waves' chunks are the latency: 8 and 4, 32
// x 64 x 2048 4.4 (one row of four waves 4.8).
template <typename XT, typename WT, bool ALIGNED>
static hipError_t rows_tile(const LinearArgs& p, int ncu, hipStream_t s) {
  const RowsPlan r = rows_plan(p.m, p.n, p.k, sizeof(XT), sizeof(WT), ncu);
  switch (r.rf * 8 + r.cf) {
    case 2 * 8 + 4: return rows_launch<XT, WT, 2, 4, 4, 2, ALIGNED>(p, s);
    case 4 * 8 + 2: return rows_launch<XT, WT, 4, 2, 4, 2, ALIGNED>(p, s);
    case 2 * 8 + 2: return rows_launch<XT, WT, 2, 2, 4, 2, ALIGNED>(p, s);
    case 2 * 8 + 1: return rows_launch<XT, WT, 2, 1, 4, 4, ALIGNED>(p, s);
    case 1 * 8 + 2: return rows_launch<XT, WT, 1, 2, 4, 4, ALIGNED>(p, s);
    default: return rows_launch<XT, WT, 1, 1, 8, 4, ALIGNED>(p, s);
  }
}

template <typename XT, typename WT>
static hipError_t rows_align(const LinearArgs& p, int ncu, hipStream_t s) {
  return p.aligned ? rows_tile<XT, WT, true>(p, ncu, s) : rows_tile<XT, WT, false>(p, ncu, s);
}

// Rows of k values of any alignment to rows of `per_row` times 16 bytes, zeros
// behind the values: 16 bytes per thread.
template <typename T>
__global__ __launch_bounds__(256) void linear_align_kernel(const T* __restrict__ src, int64_t ld, int rows, int k,
                                                           int per_row, uint4* __restrict__ dst) {
  constexpr int PER = 16 / (int)sizeof(T);
  const int i = blockIdx.x * 256 + threadIdx.x, row = i / per_row, c = (i - row * per_row) * PER;
  if (row >= rows) return;
  const T* at = src + row * ld + c;
  dst[i] = k - c >= PER ? load16<false>(at) : load16_end<false>(at, k - c);
}
template <typename T>
static hipError_t align_rows(const void* src, int64_t ld, int rows, int k, int64_t bytes, void* dst, hipStream_t s) {
  const int64_t chunks = bytes / 16;  // (of at most 512 MiB)
  linear_align_kernel<<<(unsigned)((chunks + 255) / 256), 256, 0, s>>>(reinterpret_cast<const T*>(src), ld, rows, k,
                                                                       (int)(chunks / rows), reinterpret_cast<uint4*>(dst));
  return hipGetLastError();
}

hipError_t linear_align_bf16(const void* src, int64_t ld, int rows, int k, int64_t bytes, void* dst, hipStream_t s) {
  return align_rows<uint16_t>(src, ld, rows, k, bytes, dst, s);
}

hipError_t launch_linear(const LinearArgs& p, int nwg, float* scratch, int64_t scratch_floats, hipStream_t s) {
  if (const TilesPlan t = linear_tiles_plan(p, nwg, scratch_floats); t.use) {
    LinearArgs q = p;
    char* copy = reinterpret_cast<char*>(scratch + t.cut.floats(p.n));
    q.k = t.k;
    hipError_t e = hipSuccess;
    if (t.x_bytes) {
      e = align_rows<uint16_t>(p.x, p.ldx, p.m, p.k, t.x_bytes, copy, s);
      q.x = copy;
      q.ldx = t.k;
      copy += t.x_bytes;
    }
    if (t.w_bytes && e == hipSuccess) {
      e = p.w_dtype == kFP8 ? align_rows<uint8_t>(p.w, p.ldw, p.n, p.k, t.w_bytes, copy, s)
                            : align_rows<uint16_t>(p.w, p.ldw, p.n, p.k, t.w_bytes, copy, s);
      q.w = copy;
      q.ldw = t.k;
    }
    return e == hipSuccess ? launch_linear_tiles(q, t.cut, nwg, scratch, s) : e;
  }
  if (p.w_dtype == kF32) return rows_align<float, float>(p, nwg, s);
  if (p.w_dtype == kBF16) return rows_align<uint16_t, uint16_t>(p, nwg, s);
  return rows_align<uint16_t, uint8_t>(p, nwg, s);
}

}  // namespace aep
