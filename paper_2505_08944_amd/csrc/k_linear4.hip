// Dense product with 4-bit weights (mx4.h): y = f(x W^T + b) + r, x bf16.
//
// The codes become exact bf16 values in registers (four conversions per eight
// values, the block's power among them) and go to bf16 MFMAs, so sums are those of
// a bf16 product with the same values.
//
// Row kernel: bound by the stream of W.  Tiles of 16 RF rows by 16 CF channels; the
// waves of a workgroup split K, one piece of 128 of it (k_mx4.hip) per step, and add
// their sums in LDS in wave order.  W comes in the order in which MFMA operands lie in
// lanes, 1 KB in a row per wave and load; x takes the way through the wave's own LDS
// that the other row kernel's operands take (k_linear.hip).
#include <algorithm>

#include "linear4.h"
#include "linear_epilogue.h"
#include "mx4.h"

namespace aep {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

template <bool ALIGNED>
__device__ __forceinline__ uint4 load_x(const uint16_t* __restrict__ p) {
  uint4 v;
  if constexpr (ALIGNED)
    v = *reinterpret_cast<const uint4*>(p);
  else
    __builtin_memcpy(&v, p, 16);
  return v;
}
// At the end of a row: values from `left` on are zeros.
__device__ __forceinline__ uint4 load_x_end(const uint16_t* __restrict__ p, int left) {
  uint16_t v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = j < left ? p[j] : uint16_t(0);
  uint4 o;
  __builtin_memcpy(&o, v, 16);
  return o;
}

template <int RF, int CF, int WAVES, int D, bool ALIGNED>
__global__ __launch_bounds__(WAVES * 64) void linear4_rows_kernel(const LinearArgs p) {
  constexpr int TM = RF * 16, TN = CF * 16, PITCH = TN + 4;
  constexpr int kStage = RF * 4096;      // a wave's x of a step
  constexpr int kPart = TM * PITCH * 4;  // its sums
  __shared__ __attribute__((aligned(1024))) unsigned char smem[WAVES * (kStage > kPart ? kStage : kPart)];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rr = lane & 15, hh = lane >> 4;
  // an XCD gets a contiguous run of tiles, row tiles of a column band adjacent
  const int64_t per = gridDim.x >> 3;
  const int64_t tile = (int64_t)blockIdx.y * gridDim.x + (int64_t)(blockIdx.x & 7) * per + (blockIdx.x >> 3);
  const int tm = (p.m + TM - 1) / TM, bands = (p.n + 15) / 16;
  if (tile >= (int64_t)tm * ((p.n + TN - 1) / TN)) return;
  const int ti = (int)(tile % tm), tj = (int)(tile / tm);
  const int m0 = ti * TM, n0 = tj * TN;
  const int K = p.k, steps = (K + 127) / 128, whole = K / 128;

  // x: this lane's row and 16-byte piece of a load of 16 rows by 64 bytes
  const int lr = lane >> 2, lq = (lane & 3) ^ (lane >> 4);
  const uint16_t* xr[RF];
#pragma unroll
  for (int i = 0; i < RF; ++i)
    xr[i] = reinterpret_cast<const uint16_t*>(p.x) + (int64_t)min(m0 + i * 16 + lr, p.m - 1) * p.ldx + lq * 8;
  const uint8_t* wr[CF];
#pragma unroll
  for (int j = 0; j < CF; ++j)
    wr[j] = reinterpret_cast<const uint8_t*>(p.w) + (int64_t)min(tj * CF + j, bands - 1) * steps * kLinear4Piece;

  f32x4_t acc[RF][CF];
#pragma unroll
  for (int i = 0; i < RF; ++i)
#pragma unroll
    for (int j = 0; j < CF; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  uint4 xa[D][RF][4], wa[D][CF];
  uint32_t sa[D][CF];
  auto load_w = [&](int b, int c) {
#pragma unroll
    for (int j = 0; j < CF; ++j) {
      const uint8_t* at = wr[j] + (int64_t)c * kLinear4Piece;
      wa[b][j] = *reinterpret_cast<const uint4*>(at + lane * 16);
      sa[b][j] = at[1024 + lane];
    }
  };
  auto load = [&](int b, int c) {
    load_w(b, c);
#pragma unroll
    for (int i = 0; i < RF; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) xa[b][i][q] = load_x<ALIGNED>(xr[i] + c * 128 + q * 32);
  };
  unsigned char* mine = smem + wave * kStage;
  // One wave's LDS accesses are carried out in the order in which they were issued: the
  // compiler only has to keep it, across lanes that it does not know to share values.
  auto wave_order = [&] {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  auto mma = [&](int b) {
    wave_order();
#pragma unroll
    for (int i = 0; i < RF; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) *reinterpret_cast<uint4*>(mine + (i * 4 + q) * 1024 + lane * 16) = xa[b][i][q];
    wave_order();
    // lane: k = 32 hh + 8 s .. of the step
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      uint4 x[RF];
#pragma unroll
      for (int i = 0; i < RF; ++i)
        x[i] = *reinterpret_cast<const uint4*>(mine + (i * 4 + hh) * 1024 + (rr * 4 + (s ^ (rr >> 2))) * 16);
#pragma unroll
      for (int j = 0; j < CF; ++j) {
        const uint32_t w = s == 0 ? wa[b][j].x : s == 1 ? wa[b][j].y : s == 2 ? wa[b][j].z : wa[b][j].w;
        const bf16x8_t a = __builtin_bit_cast(bf16x8_t, mx4_bf16x8(w, mx4_scale(sa[b][j])));
#pragma unroll
        for (int i = 0; i < RF; ++i)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8_t, x[i]), acc[i][j], 0, 0, 0);
      }
    }
  };

  // This wave's steps, D at a time.  No branch stands between the loads of the
  // loop, so that the wait for one step leaves the later ones in flight.
  int c = wave, n = (whole - wave + WAVES - 1) / WAVES;
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
  if (steps > whole && wave == whole % WAVES) {  // the weights are whole there, x is not
    load_w(0, whole);
#pragma unroll
    for (int i = 0; i < RF; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        xa[0][i][q] = load_x_end(xr[i] + whole * 128 + q * 32, K - whole * 128 - q * 32 - lq * 8);
    mma(0);
  }

  // lane: output row rr of a fragment, four consecutive columns 4 hh ..
  __syncthreads();  // the sums take x's place
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

template <int RF, int CF, int WAVES, int D>
static hipError_t rows4_launch(const LinearArgs& p, hipStream_t s) {
  const int64_t tiles = (int64_t)((p.m + RF * 16 - 1) / (RF * 16)) * ((p.n + CF * 16 - 1) / (CF * 16));
  // (at most 2^30 tiles; a grid's side has fewer than 2^32 threads)
  const int64_t gx = std::min<int64_t>((tiles + 7) / 8 * 8, 1 << 21);
  const dim3 grid((unsigned)gx, (unsigned)((tiles + gx - 1) / gx));
  if (p.x_aligned)
    linear4_rows_kernel<RF, CF, WAVES, D, true><<<grid, WAVES * 64, 0, s>>>(p);
  else
    linear4_rows_kernel<RF, CF, WAVES, D, false><<<grid, WAVES * 64, 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_linear4_rows(const LinearArgs& p, const RowsPlan& r, hipStream_t s) {
  switch (r.rf * 8 + r.cf) {
    case 4 * 8 + 2: return rows4_launch<4, 2, 4, 1>(p, s);
    case 2 * 8 + 2: return rows4_launch<2, 2, 8, 2>(p, s);
    case 2 * 8 + 1: return rows4_launch<2, 1, 8, 2>(p, s);
    default: return rows4_launch<1, 1, 8, 4>(p, s);
  }
}

RowsPlan rows4_plan(int m, int n, int k, int ncu) {
  constexpr int kShapes[][2] = {{4, 2}, {2, 2}, {2, 1}, {1, 1}};
  RowsPlan best{0, 0, 1e300};
  for (auto& q : kShapes) {
    const int rf = q[0], cf = q[1];
    const int64_t tiles = ((int64_t)(m + rf * 16 - 1) / (rf * 16)) * ((n + cf * 16 - 1) / (cf * 16));
    const double bytes = 16.0 * (rf * 2 + cf * 0.53) * (double)k;
    const double us = 3.0 + (double)((tiles + ncu - 1) / ncu) * bytes / 76e3;
    if (us < best.us) best = RowsPlan{rf, cf, us};
  }
  return best;
}

Linear4Plan linear4_plan(const LinearArgs& p, int nwg, int64_t max_bytes) {
  Linear4Plan r{};
  r.k8 = (p.k + 7) / 8 * 8;
  if (p.n < 8 || p.k >= 1 << 22 || std::max(p.ldy, p.res ? p.ldr : 0) >= 1 << 22) return r;
  const double rows = rows4_plan(p.m, p.n, p.k, nwg).us;
  if (rows < 16.0) return r;
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

hipError_t launch_linear4(const LinearArgs& p, int nwg, void* scratch, int64_t bytes, hipStream_t s) {
  const Linear4Plan r = linear4_plan(p, nwg, scratch ? bytes : 0);
  if (!r.widen) return launch_linear4_rows(p, rows4_plan(p.m, p.n, p.k, nwg), s);
  char* at = reinterpret_cast<char*>(scratch);
  LinearArgs q = p;
  hipError_t e = launch_linear4_unpack(reinterpret_cast<const uint8_t*>(p.w), p.n, p.k, r.k8, reinterpret_cast<uint16_t*>(at), s);
  q.w = at;
  q.ldw = q.k = r.k8;
  at += r.w_bytes;
  if (r.x_bytes && e == hipSuccess) {
    e = linear_align_bf16(p.x, p.ldx, p.m, p.k, r.x_bytes, at, s);
    q.x = at;
    q.ldx = r.k8;
    at += r.x_bytes;
  }
  if (e != hipSuccess) return e;
  const LinearPlan& t = linear_plan(p.m, p.n, r.k8, false, p.wide, nwg, (bytes - r.w_bytes - r.x_bytes) / 4);
  return launch_linear_tiles(q, t.cut, nwg, reinterpret_cast<float*>(at), s);
}

}  // namespace aep
