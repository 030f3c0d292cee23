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
// that the other row kernel's operands take (k_linear.hip).  Captured, weights from HBM (in
// brackets: from the Infinity Cache): 1 x 14336 x 4096 9.7 us (7.0; its bytes at a large
// copy's rate 6.0), 32 x 4096 x 4096 6.4 (5.5; 1.9), an empty launch 1.5.
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
template <bool ALIGNED>
__device__ __forceinline__ uint4 load_x_end(const uint16_t* __restrict__ p, int left) {
  if (left >= 8) return load_x<ALIGNED>(p);
  uint4 o = make_uint4(0, 0, 0, 0);
  if (left > 0) {
    uint16_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < left ? p[j] : uint16_t(0);
    __builtin_memcpy(&o, v, 16);
  }
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
        xa[0][i][q] = load_x_end<ALIGNED>(xr[i] + whole * 128 + q * 32, K - whole * 128 - q * 32 - lq * 8);
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

// Tile kernel, for hundreds of rows: 128 rows by 128 channels, eight waves as two groups that take every other
// step of K, each of a group's four a quarter of 64 by 64.  x goes through LDS once for a group, W's codes
// straight into the registers of the two waves that use them, so that a CU takes 32 KB of x and
// 17 of W per step: that stream from L2 is half of what its MFMAs take.  A round of
// both groups takes 3700 cycles, its MFMAs 2048: waves that wait for LDS, or at the barrier, and the conversions
// between the MFMAs are the rest (777 x 4096 x 4096 with residual 40 us; rows of 64 by 64 55, widened
// first 54).
// A row of x's step is 16 pieces of 16 bytes; piece c of row r lies at place c ^ (r % 16) of the row's 256
// bytes, so that 16 lanes that read one piece of 16 rows hit all banks.
template <bool ALIGNED>
__global__ __launch_bounds__(512, 2) void linear4_tile_kernel(const LinearArgs p) {
  constexpr int T = 128, kStage = T * 256, PITCH = T + 4;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * kStage];  // [group][2 stages]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rr = lane & 15, hh = lane >> 4, group = wave >> 2, wm = wave >> 1 & 1, wn = wave & 1;
  // an XCD gets a contiguous run of tiles, in panels of four row tiles
  const int64_t per = gridDim.x >> 3;
  const int64_t tile = (int64_t)blockIdx.y * gridDim.x + (int64_t)(blockIdx.x & 7) * per + (blockIdx.x >> 3);
  const int tm = (p.m + T - 1) / T, tn = (p.n + T - 1) / T;
  if (tile >= (int64_t)tm * tn) return;
  const int panel = (int)(tile / (4 * (int64_t)tn)), high = min(4, tm - panel * 4);
  const int in = (int)(tile - (int64_t)panel * 4 * tn), m0 = (panel * 4 + in % high) * T, n0 = in / high * T;
  const int K = p.k, steps = (K + 127) / 128, bands = (p.n + 15) / 16;

  // staging: this thread's 8 pieces of a step, of rows 16 apart
  const int t4 = tid & 255, srow = t4 >> 4, sc = t4 & 15;
  const uint8_t* x0 = reinterpret_cast<const uint8_t*>(p.x) + (int64_t)m0 * p.ldx * 2;
  uint32_t xo[8];  // (bytes from the tile's first row on: rows are below 2^22 values)
#pragma unroll
  for (int i = 0; i < 8; ++i) xo[i] = (uint32_t)min(srow + i * 16, p.m - 1 - m0) * (uint32_t)p.ldx * 2 + sc * 16;
  const auto x_at = [&](int i, int c) { return reinterpret_cast<const uint16_t*>(x0 + c * 256 + xo[i]); };
  const uint8_t* wr[4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    wr[j] = reinterpret_cast<const uint8_t*>(p.w) + (int64_t)min(n0 / 16 + wn * 4 + j, bands - 1) * steps * kLinear4Piece;

  f32x4_t acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  uint4 xa[8], wa[2][4];
  uint32_t sa[2][4];
  const auto load_x_step = [&](int c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) xa[i] = load_x<ALIGNED>(x_at(i, c));
  };
  const auto load_w_step = [&](int b, int c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint8_t* at = wr[j] + (int64_t)c * kLinear4Piece;
      wa[b][j] = *reinterpret_cast<const uint4*>(at + lane * 16);
      sa[b][j] = at[1024 + lane];
    }
  };
  unsigned char* mine = smem + group * 2 * kStage;
  const auto stage = [&](int b) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      *reinterpret_cast<uint4*>(mine + b * kStage + (srow + i * 16) * 256 + (sc ^ srow) * 16) = xa[i];
  };
  // Operands of a quarter of a step (k = 32 hh + 8 s .. of it), and its MFMAs.
  const auto read = [&](bf16x8_t* x, int b, int s) {
    const unsigned char* at = mine + b * kStage + (wm * 64 + rr) * 256 + ((hh * 4 + s) ^ rr) * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const bf16x8_t*>(at + i * (16 * 256));
  };
  const auto mma = [&](const bf16x8_t* x, int b, int s) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t w = s == 0 ? wa[b][j].x : s == 1 ? wa[b][j].y : s == 2 ? wa[b][j].z : wa[b][j].w;
      const bf16x8_t a = __builtin_bit_cast(bf16x8_t, mx4_bf16x8(w, mx4_scale(sa[b][j])));
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, x[i], acc[i][j], 0, 0, 0);
    }
  };

  // A group's steps: group, group + 2, ...; both groups pass the same barriers, and no branch stands
  // between the loads of the loop (behind the end they take the last step again, which nobody uses).
  const int whole = K / 128, last = whole - 1;
  if (whole) {
    load_x_step(min(group, last));
    load_w_step(0, min(group, last));
    stage(0);
    load_x_step(min(group + 2, last));
    __syncthreads();
    // Operands are read a quarter ahead, and what the next step needs is staged between the quarters:
    // all of it in front of them, LDS would serve nobody's operands for that long.
    const auto round = [&](int b, int i) {
      const int c = 2 * i + group;
      bf16x8_t x[2][4];
      read(x[0], b, 0);
      load_w_step(b ^ 1, min(c + 2, last));
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        __builtin_amdgcn_sched_barrier(0);
        if (s < 3) read(x[(s + 1) & 1], b, s + 1);
        if (c < whole) mma(x[s & 1], b, s);
#pragma unroll
        for (int q = 2 * s; q < 2 * s + 2; ++q) {
          // (what the place held was read before the last barrier)
          *reinterpret_cast<uint4*>(mine + (b ^ 1) * kStage + (srow + q * 16) * 256 + (sc ^ srow) * 16) = xa[q];
          xa[q] = load_x<ALIGNED>(x_at(q, min(c + 4, last)));
        }
      }
      __syncthreads();
    };
    const int rounds = (whole + 1) / 2;
    int i = 0;
    for (; i + 1 < rounds; i += 2) {
      round(0, i);
      round(1, i + 1);
    }
    if (i < rounds) round(0, i);
  }
  if (steps > whole) {  // the weights are whole there, x is not
    if (!group) {
#pragma unroll
      for (int i = 0; i < 8; ++i) xa[i] = load_x_end<ALIGNED>(x_at(i, whole), K - whole * 128 - sc * 8);
      load_w_step(0, whole);
      stage(0);
    }
    __syncthreads();
    if (!group) {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        bf16x8_t x[4];
        read(x, 0, s);
        mma(x, 0, s);
      }
    }
    __syncthreads();
  }

  // The groups' sums in x's place, rows of 128 channels; then four channels per thread.
  float* part = reinterpret_cast<float*>(smem);
  const auto place = [&](int i2, int j) {
    return reinterpret_cast<f32x4_t*>(part + (wm * 64 + i2 * 16 + rr) * PITCH + wn * 64 + j * 16 + hh * 4);
  };
  if (group) {
#pragma unroll
    for (int i2 = 0; i2 < 4; ++i2)
#pragma unroll
      for (int j = 0; j < 4; ++j) *place(i2, j) = acc[i2][j];
  }
  __syncthreads();
  if (!group) {
#pragma unroll
    for (int i2 = 0; i2 < 4; ++i2)
#pragma unroll
      for (int j = 0; j < 4; ++j) *place(i2, j) += acc[i2][j];
  }
  __syncthreads();
  // A thread has four channels of every sixteenth row; all that it loads is requested before the
  // first store, which the loads behind it would wait for.
  const int q = tid % 32 * 4, left = p.n - n0 - q, r0 = tid / 32;
  if (left <= 0) return;
  float4 bias = make_float4(0.f, 0.f, 0.f, 0.f), res[8];
  if (p.bias) bias = load4(p.bias, p.bias_dtype, n0 + q, left);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    res[e] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (p.res && m0 + r0 + e * 16 < p.m) res[e] = load4(p.res, p.res_dtype, (int64_t)(m0 + r0 + e * 16) * p.ldr + n0 + q, left);
  }
  by_fn(p.fn, [&](auto fn) {
    constexpr int FN = decltype(fn)::value;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int r = r0 + e * 16;
      const float4 v = *reinterpret_cast<const float4*>(part + r * PITCH + q);
      if (m0 + r < p.m)
        store4(p.y, p.y_dtype, (int64_t)(m0 + r) * p.ldy + n0 + q, left,
               make_float4(linear_fn<FN>(v.x + bias.x) + res[e].x, linear_fn<FN>(v.y + bias.y) + res[e].y,
                           linear_fn<FN>(v.z + bias.z) + res[e].z, linear_fn<FN>(v.w + bias.w) + res[e].w));
    }
  });
}

static hipError_t launch_linear4_tile(const LinearArgs& p, hipStream_t s) {
  const int64_t tiles = (int64_t)((p.m + 127) / 128) * ((p.n + 127) / 128);
  const int64_t gx = std::min<int64_t>((tiles + 7) / 8 * 8, 1 << 21);
  const dim3 grid((unsigned)gx, (unsigned)((tiles + gx - 1) / gx));
  if (p.x_aligned)
    linear4_tile_kernel<true><<<grid, 512, 0, s>>>(p);
  else
    linear4_tile_kernel<false><<<grid, 512, 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_linear4_rows(const LinearArgs& p, const RowsPlan& r, hipStream_t s) {
  if (r.rf == 8) return launch_linear4_tile(p, s);
  switch (r.rf * 8 + r.cf) {
    case 4 * 8 + 4: return rows4_launch<4, 4, 8, 1>(p, s);
    case 2 * 8 + 4: return rows4_launch<2, 4, 8, 1>(p, s);
    case 2 * 8 + 2: return rows4_launch<2, 2, 8, 1>(p, s);
    case 1 * 8 + 4: return rows4_launch<1, 4, 8, 1>(p, s);
    case 1 * 8 + 2: return rows4_launch<1, 2, 8, 2>(p, s);
    default: return rows4_launch<1, 1, 8, 2>(p, s);
  }
}

hipError_t launch_linear4(const LinearArgs& p, int nwg, void* scratch, int64_t bytes, hipStream_t s) {
  const Linear4Plan r = linear4_plan(p, nwg, scratch ? bytes : 0);
  if (!r.widen) return launch_linear4_rows(p, r.rows, s);
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
