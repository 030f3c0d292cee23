// Tile kernel of the dense product: y = f(s * (x W^T) + b) + r for bf16 x and
// bf16 or fp8 W whose rows are 16-byte aligned, where the matrix cores or the
// operands' way through L2 bound the product.
//
// One persistent launch, a 512-thread workgroup per CU, tiles of 256 x 256 (and
// smaller ones where rows or tiles run out, linear_tiles.h), K steps of 64.
//
// Ping-pong, as in the grouped FFN: the eight waves form two groups of four, a
// SIMD runs one wave of each, and a workgroup barrier ends every slot.  In a
// slot one group issues the MFMAs of its next phase while the other reads that
// phase's operands from LDS and issues the direct-to-LDS loads of a later K
// step.  The load stream runs on into the workgroup's next tile.
//
// What bounds it: the matrix cores, at the clock that the card's power leaves them
// (main loop of a 256 x 256 tile 1.46 .. 1.56 PFLOP/s), and below that size, by
// counters, neither they nor LDS: of 128 x 128 tiles (777 x 4096 x 4096) a CU's MFMAs
// take 38% of the cycles and its LDS reads 29%, without conflicts, while it takes 2
// MB from L2 at 55 .. 76 GB/s, three quarters of them hits.  Such a tile moves twice
// the bytes per operation, so that shape is for what is left over.  Measured: 4096 x 14336 x 4096 with bias
// and SiLU 348 .. 380 us (1.27 .. 1.38 PFLOP/s), 2048 x 4096 x 14336 fp8 189 (1.27;
// one round of 128 tiles cut in halves), 777 x 4096 x 4096 38 (0.68; 3.04 row
// tiles).  256 x 128 tiles have four waves along their rows (two: 5% longer).
//
// Rows of x past m and of W past n, and what lies between the end of a row and
// the end of its last K step, are out of the loads' range: they read as zeros.
#include <limits.h>

#include <algorithm>

#include "linear_epilogue.h"
#include "linear_tiles.h"

namespace aep {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lds_vptr;

constexpr int kTileLds = 160 * 1024;

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// A raw buffer resource over [base, base + bytes): accesses past the end read
// zeros and write nothing.
struct TileRsrc {
  int lo, hi, bytes;
  __device__ __forceinline__ i32x4_t words() const { return i32x4_t{lo, hi, bytes, 0x00020000}; }
};
__device__ __forceinline__ TileRsrc tile_rsrc(const void* base, uint32_t bytes) {
  const uint64_t a = (uint64_t)(uintptr_t)base;
  return TileRsrc{uniform((int)(uint32_t)a), uniform((int)((uint32_t)(a >> 32) & 0xFFFFu)), uniform((int)bytes)};
}

// Lane l loads the 16 bytes at voff + soff of the resource to lds_addr + 16 l.
// Inline asm, so that the compiler does not wait for it before every LDS read;
// the kernel waits itself.  It writes no register.  The wait states around it
// are checked in the built code (one after the write of M0 is here).
__device__ __forceinline__ void lds_load16(i32x4_t rsrc, uint32_t voff, uint32_t soff, uint32_t lds_addr) {
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(voff), "s"(rsrc),
               "s"(soff), "s"(__builtin_amdgcn_readfirstlane(lds_addr))
               : "memory", "m0");
}

template <int N>
__device__ __forceinline__ void wait_loads() {  // all but the last N vector memory operations
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 0xf) | ((N >> 4) << 14) | (0x7 << 4) | (0xf << 8));
}
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(0xf | (3 << 14) | (0x7 << 4)); }
__device__ __forceinline__ void slot_end() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// The launch's arguments, read again through the scalar cache where they are
// needed: kept in registers through the main loop they would not fit.
struct TileParams {
  LinearArgs a;
  LinearCut cut;
  float* scratch;
};
template <typename T>
using const_ptr = const __attribute__((address_space(4))) T*;
__device__ __forceinline__ const_ptr<TileParams> launch_params() {
  return (const_ptr<TileParams>)__builtin_amdgcn_kernarg_segment_ptr();
}
template <typename T>
__device__ __forceinline__ T read_again(const_ptr<T> at) {
  asm volatile("" : "+s"(at));
  return *(const T*)at;
}
__device__ __forceinline__ LinearArgs the_args() { return read_again<LinearArgs>(&launch_params()->a); }
__device__ __forceinline__ LinearCut the_cut() { return read_again<LinearCut>(&launch_params()->cut); }
__device__ __forceinline__ float* the_scratch() { return read_again<float*>(&launch_params()->scratch); }

// ------------------------------------------------------------------- items
// Rows [m0, ..), columns [n0, ..), K steps [k0, k0 + kn); part: where its sums
// go in the scratch (-1: to y).
struct LinearItem {
  int m0, n0, k0, kn;
  int64_t part;
};

// A tile's place among nrow x ncol: panels of 8 column tiles, row tiles one
// after another inside a panel, so that the run of tiles an XCD gets is a
// compact block whose operand bands its L2 holds.
__device__ __forceinline__ void tile_place(int nrow, int ncol, int tile, int& rt, int& ct) {
  const int per = 8 * nrow, pi = tile / per, in = tile - pi * per, w = min(8, ncol - 8 * pi);
  rt = in / w;
  ct = 8 * pi + (in - rt * w);
}

__device__ __forceinline__ LinearItem linear_item(int item) {
  const LinearCut c = the_cut();
  const int KT = (read_again<int>(&launch_params()->a.k) + 63) >> 6;
  LinearItem it;
  it.part = -1;
  int piece = 0, pieces = 1, rt, ct;
  if (item < c.whole) {
    tile_place(c.nrow, c.ncol, item, rt, ct);
    it.m0 = rt * 256;
    it.n0 = ct * 256;
  } else if (int j = item - c.whole; j < c.rest_items()) {
    pieces = c.p0;
    const int t = j / pieces;
    piece = j - t * pieces;
    tile_place(c.nrow, c.ncol, c.whole + (c.halves == 2 ? t >> 1 : t), rt, ct);
    it.m0 = rt * 256;
    it.n0 = ct * 256 + (c.halves == 2 ? (t & 1) * 128 : 0);
    if (pieces > 1) it.part = (int64_t)j * (65536 / c.halves);
  } else {
    j -= c.rest_items();
    pieces = c.pr;
    const int t = j / pieces;
    piece = j - t * pieces;
    tile_place(c.lrow, (read_again<int>(&launch_params()->a.n) + 127) / 128, t, rt, ct);
    it.m0 = c.nrow * 256 + rt * (256 >> c.fam);
    it.n0 = ct * 128;
    if (pieces > 1) it.part = c.rest_floats() + (int64_t)j * (32768 >> c.fam);
  }
  it.m0 = uniform(it.m0);
  it.n0 = uniform(it.n0);
  it.k0 = pieces == 1 ? 0 : uniform((int)((int64_t)piece * KT / pieces));
  it.kn = pieces == 1 ? KT : uniform((int)((int64_t)(piece + 1) * KT / pieces)) - it.k0;
  return it;
}

// Tile shape of an item: 0: 256 x 256, 1: 256 x 128, 2: 128 x 128, 3: 64 x 128.
__device__ __forceinline__ int linear_kind(const LinearCut& c, int item) {
  if (item < c.whole) return 0;
  return item < c.whole + c.rest_items() ? c.halves - 1 : 1 + c.fam;
}

// The workgroup's r-th item (-1: none).  An XCD gets a contiguous run of a
// round; odd rounds are dealt in reverse; a partial one over all XCDs, unless
// the round before it was a mix of shapes: then the workgroups that had its
// smaller items come first.
__device__ __forceinline__ int linear_nth(const LinearCut& c, int r, int nwg, int xcd, int xj) {
  const int base = r * nwg, cnt = c.items - base;
  if (cnt <= 0) return -1;
  const int lin = xcd * (nwg >> 3) + xj;
  const int rl = (r & 1) ? nwg - 1 - lin : lin;
  if (cnt >= nwg) return base + rl;
  if (r > 0 && linear_kind(c, base - nwg) != linear_kind(c, base - 1)) return rl < cnt ? base + rl : -1;
  const int q = (cnt + 7) >> 3, idx = xcd * q + xj;
  return xj < q && idx < cnt ? base + idx : -1;
}

// ------------------------------------------------------------- tile shapes
// A K step's stage holds the rows of x (128 bytes each) in units of up to 128
// rows (256 where there is one W unit), then NB units of 128 rows of W (128
// bytes each, 64 for fp8).  16-byte chunk c of row r sits at position c ^ (r %
// 8) (fp8 W rows: c ^ ((r / 4) % 4)), which spreads the rows that one read
// covers over the banks.
template <bool FP8, int FAM, int NB>
struct Shape {
  static constexpr int kRows = 256 >> FAM, kCols = 128 * NB;
  static constexpr bool kFour = NB == 2;               // four phases per K step, else one
  static constexpr int kUnits = kFour ? 2 : 1;         // x units per stage
  static constexpr int kUnitRows = kRows / kUnits;
  // Waves: kWM along the rows, 8 / kWM along the columns; RF 16-row fragments
  // per wave and unit, NP pairs of 16-column fragments per wave (two W units:
  // one of each).  256 x 128: four along the rows, so that a step's operands
  // are 128 KB of LDS reads and not 160.
  static constexpr int kWM = FAM == 0 && NB == 1 ? 4 : 2;
  static constexpr int NP = FAM == 0 ? 2 : NB;
  static constexpr int RF = kUnitRows / (16 * kWM);
  static __device__ __forceinline__ int row0(int wm) { return wm * (kUnitRows / kWM); }
  static __device__ __forceinline__ int pair0(int wn, int q) { return NB == 2 ? wn * 32 : wn * (NP * 32) + q * 32; }  // in its W unit
  static __device__ __forceinline__ int col0(int wn, int q) { return (NB == 2 ? q * 128 : 0) + pair0(wn, q); }
  static constexpr int kX = kUnitRows * 128, kW = 128 * (FP8 ? 64 : 128);
  static constexpr int kStage = kUnits * kX + NB * kW;
  static constexpr int kStages = NB == 2 ? (FP8 ? 3 : 2) : FAM == 0 ? (FP8 ? 4 : 3) : FAM == 1 ? (FP8 ? 6 : 5) : (FP8 ? 8 : 6);
  static constexpr int kLX = kUnitRows / 64, kLW = FP8 ? 1 : 2;  // loads per wave and unit
  static_assert(kStages * kStage <= kTileLds, "the ring fits the LDS");
};

// Which item's which K step the next stage is filled from.  A last K step that
// is not whole (tail) comes on its own, with other offsets.
struct TileStream {
  TileRsrc x, w;
  int k, step, left, tail;
};

template <bool FP8, int FAM, int NB>
__device__ __forceinline__ void stream_to(TileStream& st, const LinearItem& it) {
  using S = Shape<FP8, FAM, NB>;
  constexpr int es = FP8 ? 1 : 2;
  const LinearArgs p = the_args();
  // (the second half of the last tile may lie past the matrix: it reads the last row, and nothing is stored)
  const int n0 = min(it.n0, p.n - 1);
  const int rows = min(p.m - it.m0, S::kRows), cols = min(p.n - n0, S::kCols);
  st.x = tile_rsrc(reinterpret_cast<const uint16_t*>(p.x) + (int64_t)it.m0 * p.ldx,
                   ((uint32_t)(rows - 1) * (uint32_t)p.ldx + (uint32_t)p.k) * 2u);
  st.w = tile_rsrc(reinterpret_cast<const unsigned char*>(p.w) + (int64_t)n0 * p.ldw * es,
                   ((uint32_t)(cols - 1) * (uint32_t)p.ldw + (uint32_t)p.k) * es);
  st.k = it.k0;
  st.step = 1;
  st.tail = (p.k & 63) && it.k0 + it.kn == (p.k + 63) >> 6 ? 1 : 0;
  st.left = it.kn - st.tail;
}
__device__ __forceinline__ void stream_end(TileStream& st) {
  // nothing more: every lane is out of range (the scalar offset stays 0)
  st.x.bytes = st.w.bytes = 0;
  st.k = st.step = st.tail = 0;
  st.left = INT_MAX;
}

// Four consecutive values of the bias or the scales from column c on (clamped:
// n is at least 4), whatever their alignment.
__device__ __forceinline__ f32x4_t columns4(const void* v, int dtype, int c, int n) {
  c = min(c, n - 4);
  if (dtype == kF32) {
    f32x4_t o;
    __builtin_memcpy(&o, reinterpret_cast<const float*>(v) + c, 16);
    return o;
  }
  uint2 w;
  __builtin_memcpy(&w, reinterpret_cast<const uint16_t*>(v) + c, 8);
  return f32x4_t{bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y)};
}

// The epilogue of a finished tile: scale, bias, activation, residual and one
// rounding, from the registers.  A lane holds columns 16 j + 4 hh .. + 3 of
// fragment (i, j)'s row rr.
//
// Everything that is loaded is requested before the first store, and stores
// are never waited for: vector memory operations complete in order, so a load
// behind the stores would wait for them and for the operand ring as well.
// (With loads between the stores, and the activation chosen value by value, a
// 256 x 256 tile's epilogue took 24 us: 4096 x 14336 x 4096 with bias and SiLU
// 461 us, now 348.)
//
// Wide results (bf16, aligned rows of a multiple of 8 columns) go out in 16
// bytes: a swap of odd and even 16-lane rows between the two column fragments
// gives a lane 8 consecutive columns, 16 (hh & 1) + 8 (hh >> 1) on; the
// residual comes in the same way, swapped back.  Rows and columns past the
// matrix are out of the resources' range.
template <bool FP8, int FAM, int NB>
__device__ __forceinline__ void finish_wide(const LinearItem& it, int wm, int wn, int rr, int hh,
                                            f32x4_t (&acc)[Shape<FP8, FAM, NB>::kUnits][Shape<FP8, FAM, NB>::NP][Shape<FP8, FAM, NB>::RF][2]) {
  using S = Shape<FP8, FAM, NB>;
  constexpr int RF = S::RF, NU = S::kUnits, NP = S::NP;
  const LinearArgs p = the_args();
  const int rows = min(p.m - it.m0, S::kRows), cols = p.n - it.n0;
  if (cols <= 0) return;
  const uint32_t ybytes = ((uint32_t)(rows - 1) * (uint32_t)p.ldy + (uint32_t)cols) * 2u;
  __amdgpu_buffer_rsrc_t ry = __builtin_amdgcn_make_buffer_rsrc(
      reinterpret_cast<uint16_t*>(p.y) + (int64_t)it.m0 * p.ldy + it.n0, 0, (int)ybytes, 0x00020000);
  const int row = S::row0(wm) + rr;
  uint32_t yo[NP], ro[NP];  // (2^31: past any range, which is below it, with any row added)
  f32x4_t b4[NP][2], s4[FP8 ? NP : 1][2];
#pragma unroll
  for (int b = 0; b < NP; ++b) {
    const int c8 = S::col0(wn, b) + (hh & 1) * 16 + (hh >> 1) * 8;
    yo[b] = c8 < cols ? ((uint32_t)row * (uint32_t)p.ldy + (uint32_t)c8) * 2u : 0x80000000u;
    ro[b] = c8 < cols ? ((uint32_t)row * (uint32_t)p.ldr + (uint32_t)c8) * 2u : 0x80000000u;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int c = it.n0 + S::col0(wn, b) + j * 16 + hh * 4;
      b4[b][j] = p.bias ? columns4(p.bias, p.bias_dtype, c, p.n) : f32x4_t{0.f, 0.f, 0.f, 0.f};
      if constexpr (FP8) s4[b][j] = columns4(p.scale, kBF16, c, p.n);
    }
  }
  const uint32_t ystep = (uint32_t)p.ldy * 2u, rstep = (uint32_t)p.ldr * 2u;
  __amdgpu_buffer_rsrc_t rr_ = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint16_t*>(reinterpret_cast<const uint16_t*>(p.res)) + (p.res ? (int64_t)it.m0 * p.ldr + it.n0 : 0), 0,
      p.res ? (int)(((uint32_t)(rows - 1) * (uint32_t)p.ldr + (uint32_t)cols) * 2u) : 0, 0x00020000);
  auto load_res = [&](u32x4_t (&res)[RF], int u, int b) {
#pragma unroll
    for (int i = 0; i < RF; ++i)
      res[i] = __builtin_amdgcn_raw_buffer_load_b128(rr_, ro[b] + (uint32_t)(u * 128 + i * 16) * rstep, 0, 0);
  };
  by_fn(p.fn, [&](auto fn) {
    u32x4_t res[2][RF];  // the unit's residual and the next one's
    if (p.res) load_res(res[0], 0, 0);
#pragma unroll
    for (int q = 0; q < NU * NP; ++q) {
      const int u = q / NP, b = q % NP;
      if (p.res && q + 1 < NU * NP) load_res(res[(q + 1) & 1], (q + 1) / NP, (q + 1) % NP);
#pragma unroll
      for (int i = 0; i < RF; ++i) {
        float o[2][4];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float v = acc[u][b][i][j][e];
            if constexpr (FP8) v *= s4[b][j][e];
            o[j][e] = linear_fn_tile<fn()>(v + b4[b][j][e]);
          }
        if (p.res) {
          const u32x4_t v = res[q & 1][i];
          const auto s0 = __builtin_amdgcn_permlane16_swap(v[0], v[2], false, false);
          const auto s1 = __builtin_amdgcn_permlane16_swap(v[1], v[3], false, false);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            o[j][0] += bf16_lo(s0[j]);
            o[j][1] += bf16_hi(s0[j]);
            o[j][2] += bf16_lo(s1[j]);
            o[j][3] += bf16_hi(s1[j]);
          }
        }
        const auto s0 = __builtin_amdgcn_permlane16_swap(bf16_pair(o[0][0], o[0][1]), bf16_pair(o[1][0], o[1][1]), false,
                                                         false);
        const auto s1 = __builtin_amdgcn_permlane16_swap(bf16_pair(o[0][2], o[0][3]), bf16_pair(o[1][2], o[1][3]), false,
                                                         false);
        const u32x4_t w = {(unsigned)s0[0], (unsigned)s1[0], (unsigned)s0[1], (unsigned)s1[1]};
        __builtin_amdgcn_raw_buffer_store_b128(w, ry, yo[b] + (uint32_t)(u * 128 + i * 16) * ystep, 0, 0);
      }
    }
  });
}

// The same for f32 results of a multiple of 4 columns, which go out as a lane
// holds them.  The residual may be f32, or bf16 of dword-aligned rows.  (4096 x
// 4096 x 1024 with bias, SiLU and f32 residual 56 us, 26 of them its bytes and 5 the
// activation to f32's accuracy; with the short form of bf16 results 51, and that by
// finish_any 61.)
template <bool FP8, int FAM, int NB>
__device__ __forceinline__ void finish_f32(const LinearItem& it, int wm, int wn, int rr, int hh,
                                           f32x4_t (&acc)[Shape<FP8, FAM, NB>::kUnits][Shape<FP8, FAM, NB>::NP][Shape<FP8, FAM, NB>::RF][2]) {
  using S = Shape<FP8, FAM, NB>;
  constexpr int RF = S::RF, NU = S::kUnits, NP = S::NP;
  const LinearArgs p = the_args();
  const int rows = min(p.m - it.m0, S::kRows), cols = p.n - it.n0;
  if (cols <= 0) return;
  __amdgpu_buffer_rsrc_t ry = __builtin_amdgcn_make_buffer_rsrc(
      reinterpret_cast<float*>(p.y) + (int64_t)it.m0 * p.ldy + it.n0, 0,
      (int)(((uint32_t)(rows - 1) * (uint32_t)p.ldy + (uint32_t)cols) * 4u), 0x00020000);
  const uint32_t rs = p.res_dtype == kF32 ? 4u : 2u;
  __amdgpu_buffer_rsrc_t rr_ = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<char*>(reinterpret_cast<const char*>(p.res)) + (p.res ? ((int64_t)it.m0 * p.ldr + it.n0) * rs : 0), 0,
      p.res ? (int)(((uint32_t)(rows - 1) * (uint32_t)p.ldr + (uint32_t)cols) * rs) : 0, 0x00020000);
  const uint32_t ystep = (uint32_t)p.ldy * 4u, rstep = (uint32_t)p.ldr * rs;
  by_fn(p.fn, [&](auto fn) {
#pragma unroll
    for (int q = 0; q < NU * NP; ++q) {
      const int u = q / NP, b = q % NP;
      int row = S::row0(wm) + rr, c0 = hh * 4;
      asm volatile("" : "+v"(row), "+v"(c0));  // offsets are made here, not kept for all pairs
      uint32_t yo[2], ro[2];
      f32x4_t b4[2], s4[FP8 ? 2 : 1];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int c = S::col0(wn, b) + j * 16 + c0;
        yo[j] = c < cols ? (uint32_t)(row + u * 128) * ystep + (uint32_t)c * 4u : 0x80000000u;
        ro[j] = c < cols ? (uint32_t)(row + u * 128) * rstep + (uint32_t)c * rs : 0x80000000u;
        b4[j] = p.bias ? columns4(p.bias, p.bias_dtype, it.n0 + c, p.n) : f32x4_t{0.f, 0.f, 0.f, 0.f};
        if constexpr (FP8) s4[j] = columns4(p.scale, kBF16, it.n0 + c, p.n);
      }
      u32x4_t res[RF][2];
      if (p.res) {
#pragma unroll
        for (int i = 0; i < RF; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const uint32_t at = ro[j] + (uint32_t)(i * 16) * rstep;
            if (rs == 4u) {
              res[i][j] = __builtin_amdgcn_raw_buffer_load_b128(rr_, at, 0, 0);
            } else {
              const auto h = __builtin_amdgcn_raw_buffer_load_b64(rr_, at, 0, 0);
              res[i][j] = u32x4_t{h[0], h[1], 0u, 0u};
            }
          }
      }
#pragma unroll
      for (int i = 0; i < RF; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          f32x4_t v = acc[u][b][i][j];
          if constexpr (FP8) v *= s4[j];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = linear_fn<fn()>(v[e] + b4[j][e]);
          if (p.res) {
            const u32x4_t t = res[i][j];
            v += rs == 4u ? __builtin_bit_cast(f32x4_t, t) : f32x4_t{bf16_lo(t[0]), bf16_hi(t[0]), bf16_lo(t[1]), bf16_hi(t[1])};
          }
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), ry, yo[j] + (uint32_t)(i * 16) * ystep, 0, 0);
        }
      __builtin_amdgcn_sched_barrier(0);  // the next pair's values would not fit beside these
    }
  });
}

// The same for any other result: rows of any alignment and length, by unaligned
// accesses of four values.  (bf16 rows of 4097 elements, otherwise as above: 66 us,
// wide rows 41; value by value a quarter longer.)
template <bool FP8, int FAM, int NB>
__device__ __forceinline__ void finish_any(const LinearItem& it, int wm, int wn, int rr, int hh,
                                           f32x4_t (&acc)[Shape<FP8, FAM, NB>::kUnits][Shape<FP8, FAM, NB>::NP][Shape<FP8, FAM, NB>::RF][2]) {
  using S = Shape<FP8, FAM, NB>;
  constexpr int RF = S::RF, NU = S::kUnits, NP = S::NP;
  // two fragments of one x unit and pair of columns at a time: the code is long, and
  // more values would not fit beside the sums
  constexpr int RH = 2, NH = RF / RH;
#pragma unroll 1
  for (int h = 0; h < NU * NP * NH; ++h) {
    const int q = h / NH;
    f32x4_t v[RH][2];
#pragma unroll
    for (int a = 0; a < NU * NP * NH; ++a)
      if (h == a) {
#pragma unroll
        for (int i = 0; i < RH; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) v[i][j] = acc[a / NH / NP][a / NH % NP][a % NH * RH + i][j];
      }
    const LinearArgs p = the_args();
    const int m = it.m0 + (q / NP) * 128 + S::row0(wm) + h % NH * (RH * 16) + rr, n0 = it.n0 + S::col0(wn, q % NP) + hh * 4;
    // all columns of the pair lie in the matrix (or some do not)
    const bool full = it.n0 + S::col0(wn, q % NP) + 32 <= p.n;
    f32x4_t res[RH][2], b4[2];
#pragma unroll
    for (int i = 0; i < RH; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) res[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (p.res && full) {
      // (rows past the matrix: its last one)
      auto load = [&](auto dtype) {
#pragma unroll
        for (int i = 0; i < RH; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float4 t = load4(p.res, dtype(), (int64_t)min(m + 16 * i, p.m - 1) * p.ldr + n0 + j * 16, 4);
            res[i][j] = f32x4_t{t.x, t.y, t.z, t.w};
          }
      };
      if (p.res_dtype == kF32)
        load(std::integral_constant<int, kF32>{});
      else
        load(std::integral_constant<int, kBF16>{});
    } else if (p.res) {
#pragma unroll
      for (int i = 0; i < RH; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int c = n0 + j * 16;
          if (m + 16 * i < p.m && c < p.n) {
            const float4 t = load4(p.res, p.res_dtype, (int64_t)(m + 16 * i) * p.ldr + c, p.n - c);
            res[i][j] = f32x4_t{t.x, t.y, t.z, t.w};
          }
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int c = n0 + j * 16;
      const float4 t = p.bias ? load4(p.bias, p.bias_dtype, c, p.n - c) : make_float4(0.f, 0.f, 0.f, 0.f);
      b4[j] = f32x4_t{t.x, t.y, t.z, t.w};
      if constexpr (FP8) {
        const float4 s = load4(p.scale, kBF16, c, p.n - c);
#pragma unroll
        for (int i = 0; i < RH; ++i) v[i][j] *= f32x4_t{s.x, s.y, s.z, s.w};
      }
    }
    by_fn(p.fn, [&](auto fn) {
      if (p.y_dtype == kF32) {
#pragma unroll
        for (int i = 0; i < RH; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i][j][e] = linear_fn<fn()>(v[i][j][e] + b4[j][e]) + res[i][j][e];
      } else {
#pragma unroll
        for (int i = 0; i < RH; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i][j][e] = linear_fn_tile<fn()>(v[i][j][e] + b4[j][e]) + res[i][j][e];
      }
    });
    auto store = [&](auto dtype, auto all) {
#pragma unroll
      for (int i = 0; i < RH; ++i)
        if (m + 16 * i < p.m) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int c = n0 + j * 16;
            if (all() || c < p.n)
              store4(p.y, dtype(), (int64_t)(m + 16 * i) * p.ldy + c, all() ? 4 : p.n - c,
                     make_float4(v[i][j][0], v[i][j][1], v[i][j][2], v[i][j][3]));
          }
        }
    };
    using std::integral_constant;
    if (p.y_dtype == kF32)
      full ? store(integral_constant<int, kF32>{}, std::true_type{}) : store(integral_constant<int, kF32>{}, std::false_type{});
    else
      full ? store(integral_constant<int, kBF16>{}, std::true_type{}) : store(integral_constant<int, kBF16>{}, std::false_type{});
  }
}

// Runs the workgroup's chain of items of one shape from `item`, its r-th, on;
// leaves r and item at the first of another shape.
template <bool FP8, int FAM, int NB>
__device__ __forceinline__ void run_shape(unsigned char* smem, uint32_t lds_base, int nwg, int xcd, int xj, int& r,
                                          int& item) {
  using S = Shape<FP8, FAM, NB>;
  constexpr bool kFour = S::kFour;
  constexpr int RF = S::RF, NU = S::kUnits, NP = S::NP, NST = S::kStages;
  constexpr int kKind = NB == 2 ? 0 : 1 + FAM;
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));  // per-lane offsets are made here, not kept through other shapes' loops
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % S::kWM, wn = wave / S::kWM, grp = wave >> 2;
  const int rr = lane & 15, hh = lane >> 4;

  // loader offsets, the same for every tile and K step (the resources and the
  // scalar offset move); on a K step that is not whole, the lanes whose chunk
  // lies past the row's end are sent out of range
  uint32_t xoff[NU][S::kLX], woff[NB][S::kLW];
  auto set_offsets = [&](bool tail) {
    const LinearArgs p = the_args();
    const int have = tail ? p.k & 63 : 64;
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int i = 0; i < S::kLX; ++i) {
        const int row = (wave * S::kLX + i) * 8 + (lane >> 3), c = (lane & 7) ^ (lane >> 3);
        xoff[u][i] = (uint32_t)(u * 128 + row) * (uint32_t)p.ldx * 2u + (uint32_t)(c << 4);
        if (c * 8 >= have) xoff[u][i] = 0xfffffff0u;
      }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < S::kLW; ++i) {
        const int lr = wave * 16 + (FP8 ? (lane >> 2) : i * 8 + (lane >> 3));
        const int c = FP8 ? ((lane & 3) ^ ((lr >> 2) & 3)) : ((lane & 7) ^ (lr & 7));
        woff[b][i] = (uint32_t)(b * 128 + lr) * (uint32_t)p.ldw * (FP8 ? 1u : 2u) + (uint32_t)(c << 4);
        if (c * (FP8 ? 16 : 8) >= have) woff[b][i] = 0xfffffff0u;
      }
  };
  const uint32_t lx = lds_base + wave * (S::kLX * 1024), lw = lds_base + NU * S::kX + wave * (S::kLW * 1024);

  TileStream st;
  auto load_x = [&](int u, int stage) {
#pragma unroll
    for (int i = 0; i < S::kLX; ++i)
      lds_load16(st.x.words(), xoff[u][i], (uint32_t)st.k * 128u, lx + stage * S::kStage + u * S::kX + i * 1024);
  };
  auto load_w = [&](int b, int stage) {
#pragma unroll
    for (int i = 0; i < S::kLW; ++i)
      lds_load16(st.w.words(), woff[b][i], (uint32_t)st.k * (FP8 ? 64u : 128u),
                 lw + stage * S::kStage + b * S::kW + i * 1024);
  };
  auto next_k = [&] {
    --st.left;
    st.k += st.step;
  };
  // the stream has no whole K step left: the tail, if there is one
  auto to_tail = [&] {
    if (!st.tail) return false;
    st.tail = 0;
    st.left = 1;
    set_offsets(true);
    return true;
  };

  // Operands and accumulators [x unit][column pair][row fragment][column].
  // MFMA rows are W's: a lane holds four consecutive output columns of one row.
  bf16x8_t rx[RF][2], rw[NP][2][2];
  uint4 rn[FP8 && !kFour ? NP : 1][2][FP8 ? 1 : 2];  // W as read, where it becomes rw in widen()
  f32x4_t acc[NU][NP][RF][2];
  const int wrow = S::row0(wm) + rr;
  auto read_x = [&](int u, int stage) {
    const unsigned char* q = smem + stage * S::kStage + u * S::kX + wrow * 128;
#pragma unroll
    for (int i = 0; i < RF; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int c = FP8 ? 2 * hh + k : 4 * k + hh;
        rx[i][k] = *reinterpret_cast<const bf16x8_t*>(q + i * 2048 + ((c ^ (rr & 7)) << 4));
      }
  };
  auto read_w = [&](int b, int stage, bool aside) {
    const unsigned char* q = smem + stage * S::kStage + NU * S::kX + (NB == 2 ? b : 0) * S::kW;
    const int n = kFour ? 0 : b;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int lr = S::pair0(wn, b) + j * 16 + rr;
      if constexpr (FP8) {
        rn[n][j][0] = *reinterpret_cast<const uint4*>(q + lr * 64 + ((hh ^ ((rr >> 2) & 3)) << 4));
      } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint4 v = *reinterpret_cast<const uint4*>(q + lr * 128 + (((4 * k + hh) ^ (rr & 7)) << 4));
          if (aside)
            rn[0][j][k] = v;
          else
            rw[b][j][k] = __builtin_bit_cast(bf16x8_t, v);
        }
      }
    }
  };
  auto widen = [&](int b, bool aside) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if constexpr (FP8) {
        const uint4 v = rn[kFour ? 0 : b][j][0];
        const uint2 w0 = e4m3x4_to_bf16x4(v.x), w1 = e4m3x4_to_bf16x4(v.y);
        const uint2 w2 = e4m3x4_to_bf16x4(v.z), w3 = e4m3x4_to_bf16x4(v.w);
        rw[b][j][0] = __builtin_bit_cast(bf16x8_t, make_uint4(w0.x, w0.y, w1.x, w1.y));
        rw[b][j][1] = __builtin_bit_cast(bf16x8_t, make_uint4(w2.x, w2.y, w3.x, w3.y));
      } else if (aside) {
#pragma unroll
        for (int k = 0; k < 2; ++k) rw[b][j][k] = __builtin_bit_cast(bf16x8_t, rn[0][j][k]);
      }
    }
  };
  auto mma = [&](int u, int b) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < RF; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          acc[u][b][i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(rw[b][j][k], rx[i][k], acc[u][b][i][j], 0, 0, 0);
  };
  auto clear = [&] {
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int b = 0; b < NP; ++b)
#pragma unroll
        for (int i = 0; i < RF; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[u][b][i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  };

  LinearItem cur = linear_item(item), nxt = cur;
  bool has_next = false;  // the stream has moved on to nxt, item nitem
  int nitem = -1;
  stream_to<FP8, FAM, NB>(st, cur);
  set_offsets(false);

  __syncthreads();
  int stage = 0;
  // Loads in flight after the wait of a phase.  Four phases per step: those of
  // the last 4 NST - 2 phases; else NST - 2 steps.
  constexpr int kFlight = kFour ? (2 * NST - 1) * (S::kLX + S::kLW) : (NST - 2) * (S::kLX + NB * S::kLW);
  constexpr int kAhead = kFour ? NST : NST - 1;  // steps the stream is ahead
  for (int s = 0; s < kAhead; ++s) {
    if (st.left == 0 && !to_tail()) stream_end(st);
    load_w(0, s);
    load_x(0, s);
    if constexpr (NB == 2) load_w(1, s);
    if constexpr (NU == 2) load_x(1, s);
    next_k();
  }
  wait_loads<kFlight>();
  slot_end();
  if constexpr (kFour) {
    read_w(0, 0, true);
    // the first phase refills this unit, each wave for another one's reads too
    wait_lds();
    slot_end();
  }
  if (grp == 1) slot_end();

  int t = cur.kn;
  clear();
  for (;;) {
    if (st.left == 0 && !to_tail()) {
      // The stream follows the chain if this item is long enough that it is
      // at most one item ahead.
      const int ni = !has_next && cur.kn > 2 * NST ? linear_nth(the_cut(), r + 1, nwg, xcd, xj) : -1;
      if (ni >= 0 && linear_kind(the_cut(), ni) == kKind) {
        nxt = linear_item(ni);
        nitem = ni;
        has_next = true;
        stream_to<FP8, FAM, NB>(st, nxt);
        set_offsets(false);
      } else {
        stream_end(st);
      }
    }
    int seg = min(t, st.left);
    t -= seg;
    do {
      const int ns = stage + 1 == NST ? 0 : stage + 1;
      if constexpr (kFour) {
        // One phase per (x unit, W unit), in an order in which each needs one
        // new unit; a phase's loads refill the unit read one phase earlier.
#define TILE_PHASE(READS, LOADS, WIDEN, MMA) \
  do {                                       \
    READS;                                   \
    LOADS;                                   \
    wait_loads<kFlight>();                   \
    wait_lds();                              \
    WIDEN;                                   \
    slot_end();                              \
    MMA;                                     \
    slot_end();                              \
  } while (0)
        TILE_PHASE(read_x(0, stage), load_w(0, stage), widen(0, true), mma(0, 0));
        TILE_PHASE(read_w(1, stage, false), load_x(0, stage), widen(1, false), mma(0, 1));
        TILE_PHASE(read_x(1, stage), load_w(1, stage), (void)0, mma(1, 1));
        TILE_PHASE(read_w(0, ns, true), load_x(1, stage); next_k(), (void)0, mma(1, 0));
#undef TILE_PHASE
      } else {
        const int fs = stage == 0 ? NST - 1 : stage - 1;
        read_x(0, stage);
#pragma unroll
        for (int q = 0; q < NP; ++q) read_w(q, stage, false);
        load_x(0, fs);
        load_w(0, fs);
        next_k();
        wait_loads<kFlight>();
        wait_lds();
        slot_end();
        // fp8 W is widened between the MFMAs: the other slot, of reads, is the longer one
        // (2048 x 4096 x 14336 in halves 224 -> 203 us, 1024 rows of 128 144 -> 132;
        // with four phases per step it makes no difference)
#pragma unroll
        for (int q = 0; q < NP; ++q) {
          widen(q, false);
          mma(0, q);
        }
        slot_end();
      }
      stage = ns;
    } while (--seg);
    if (t > 0) continue;

    // Epilogue, from the registers.
    if (cur.part >= 0) {
      float* part = the_scratch() + cur.part;
      // a piece: its f32 sums, row by row of the tile
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int b = 0; b < NP; ++b)
#pragma unroll
          for (int i = 0; i < RF; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const int row = u * 128 + S::row0(wm) + i * 16 + rr, col = S::col0(wn, b) + j * 16 + hh * 4;
              *reinterpret_cast<f32x4_t*>(part + row * S::kCols + col) = acc[u][b][i][j];
            }
    } else if (const int wide = read_again<int>(&launch_params()->a.wide); wide == kWideBf16) {
      finish_wide<FP8, FAM, NB>(cur, wm, wn, rr, hh, acc);
    } else if (wide == kWideF32) {
      finish_f32<FP8, FAM, NB>(cur, wm, wn, rr, hh, acc);
    } else {
      finish_any<FP8, FAM, NB>(cur, wm, wn, rr, hh, acc);
    }

    r += 1;
    if (!has_next) {
      item = linear_nth(the_cut(), r, nwg, xcd, xj);
      if (grp == 0) slot_end();  // the groups are in step again
      wait_loads<0>();           // no load still targets the ring
      return;
    }
    item = nitem;
    cur = nxt;
    has_next = false;
    t = cur.kn;
    clear();
  }
}

template <bool FP8>
__global__ __launch_bounds__(512, 2) void linear_tiles_kernel(const TileParams) {  // read by launch_params()
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kTileLds];
  const uint32_t lds_base = (uint32_t)(uintptr_t)(lds_vptr)smem;
  const int nwg = gridDim.x, xcd = blockIdx.x & 7, xj = blockIdx.x >> 3;
  int r = 0;
  int item = linear_nth(the_cut(), r, nwg, xcd, xj);
  while (item >= 0) {
    const int kind = linear_kind(the_cut(), item);
    if (kind == 0)
      run_shape<FP8, 0, 2>(smem, lds_base, nwg, xcd, xj, r, item);
    else if (kind == 1)
      run_shape<FP8, 0, 1>(smem, lds_base, nwg, xcd, xj, r, item);
    else if (kind == 2)
      run_shape<FP8, 1, 1>(smem, lds_base, nwg, xcd, xj, r, item);
    else
      run_shape<FP8, 2, 1>(smem, lds_base, nwg, xcd, xj, r, item);
  }
}

// Adds the pieces' sums of the cut tiles, in piece order, and finishes them:
// 256 threads per 16 rows of a tile or half.
__global__ __launch_bounds__(256) void linear_sums_kernel(const LinearArgs p, const LinearCut c, const float* scratch) {
  int b = blockIdx.x;
  int m0, n0, rows, cols, pieces;
  const float* s = scratch;
  const int rest_blocks = c.p0 > 1 ? c.rest_parts() * 16 : 0;
  int strip;
  if (b < rest_blocks) {
    const int t = b >> 4;
    strip = b & 15;
    int rt, ct;
    tile_place(c.nrow, c.ncol, c.whole + (c.halves == 2 ? t >> 1 : t), rt, ct);
    m0 = rt * 256;
    n0 = ct * 256 + (c.halves == 2 ? (t & 1) * 128 : 0);
    rows = 256;
    cols = 256 / c.halves;
    pieces = c.p0;
    s += (int64_t)t * pieces * rows * cols;
  } else {
    b -= rest_blocks;
    const int per = 16 >> c.fam, t = b / per;
    strip = b - t * per;
    int rt, ct;
    tile_place(c.lrow, (p.n + 127) / 128, t, rt, ct);
    m0 = c.nrow * 256 + rt * (256 >> c.fam);
    n0 = ct * 128;
    rows = 256 >> c.fam;
    cols = 128;
    pieces = c.pr;
    s += c.rest_floats() + (int64_t)t * pieces * rows * cols;
  }
  const int q = cols / 4;
  for (int e = threadIdx.x; e < 16 * q; e += 256) {
    const int row = strip * 16 + e / q, col = (e % q) * 4;
    if (m0 + row >= p.m || n0 + col >= p.n) continue;
    const float* at = s + row * cols + col;
    float4 v = *reinterpret_cast<const float4*>(at);
    for (int i = 1; i < pieces; ++i) {
      const float4 a = *reinterpret_cast<const float4*>(at + (int64_t)i * rows * cols);
      v = make_float4(v.x + a.x, v.y + a.y, v.z + a.z, v.w + a.w);
    }
    linear_out4(p, m0 + row, n0 + col, p.n - n0 - col, v);
  }
}

hipError_t launch_linear_tiles(const LinearArgs& p, const LinearCut& c, int nwg, float* scratch, hipStream_t s) {
  const TileParams t{p, c, scratch};
  if (p.w_dtype == kFP8)
    linear_tiles_kernel<true><<<nwg, 512, 0, s>>>(t);
  else
    linear_tiles_kernel<false><<<nwg, 512, 0, s>>>(t);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int blocks = (c.p0 > 1 ? c.rest_parts() * 16 : 0) + (c.pr > 1 ? c.last_tiles(p.n) * (16 >> c.fam) : 0);
  if (!blocks) return hipSuccess;
  linear_sums_kernel<<<blocks, 256, 0, s>>>(p, c, scratch);
  return hipGetLastError();
}

}  // namespace aep
