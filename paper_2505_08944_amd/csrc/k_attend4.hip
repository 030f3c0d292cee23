// Attention over a paged cache of keys and values in 4 bits (cache4.h): for each row
// of queries o = sum_t p_t v_t / sum_t p_t, p_t = e^(scale q k_t), over the tokens that
// it sees, in one pass with a running reference for the exponents.
//
// A column is a row of queries and one of the heads that share a head of the cache.
// Scores are K q^T on MFMAs (rows: tokens, columns: queries), which leaves a lane 8 of 32 tokens
// of its column in the order in which it holds them as an operand of V^T p^T: the weights
// need no way through LDS.  Codes become exact bf16 in registers; p is rounded to bf16
// once, for the second product, and its sum is that of the rounded values (an MFMA with ones), so
// that weights sum to 1.  Scores, sums and references are f32.
//
// Few columns (attend4_kernel): a wave takes 32 tokens for a tile of 16 or 32 columns.
// Bound by the cache's bytes: 64 sequences of up to 16384 tokens, 8 heads of 128, 104 us
// of kernel for 507 MB (4.9 TB/s; a large copy 5.2); one sequence of 100003 tokens 24 us for 109 MB.
// Many columns (attend4_wide_kernel): four waves with 32 columns each share what they
// widen.  Of 4 x 509 rows to up to 8192 tokens (188 us with the join) MFMAs are busy in 37% of the SIMDs'
// cycles and VALU in 40%, and waves wait for 25% of their time.
//
// The work is divided evenly: all units of 128 tokens of all tiles in a row, an equal share
// for each workgroup.  Tiles that several workgroups share leave parts in the scratch, which a
// second launch joins in the order of the tokens: no atomics, equal calls give equal bits.
#include <algorithm>
#include <climits>
#include <cmath>

#include "cache4.h"
#include "linear_epilogue.h"

namespace aep {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

namespace {

using Shared = Attend4Args::Shared;
static_assert(sizeof(Shared) == kAttendShared);

constexpr int kUnit = kAttendUnit;
constexpr float kNegInf = -INFINITY;
// A column's reference is its largest score (in powers of two) and this much more when it is set, and
// holds until a weight reaches 2: few blocks change it, and no maximum is needed to see that.
constexpr float kAhead = 6.f;

// A sequence's units: tiles of columns for each head, units of tokens for each tile.
struct SeqUnits {
  SeqRows s;
  int first, nb, ct;  // first unit, units of a tile, tiles of a head
  __device__ int units(int heads) const { return heads * ct * nb; }
};
template <int COLS>
__device__ __forceinline__ SeqUnits seq_units(const Attend4Args& a, const SeqRows& s) {
  SeqUnits u;
  u.s = s;
  u.first = 0;
  if (a.window) u.first = max(0, s.len - s.n - a.window + 1) / kUnit;
  u.nb = max(1, (s.len + kUnit - 1) / kUnit - u.first);
  const int cols = s.n * a.group;
  u.ct = cols > a.over && cols <= a.most ? (cols + COLS - 1) / COLS : 0;
  return u;
}

// Where a workgroup is among the units.
struct Place {
  int w, workers;  // its number, of so many that have units
  int total;     // units of all sequences
  int u0, u1;    // this workgroup's
  int b, before; // sequence of u0, units before that sequence
  SeqRows s;     // that sequence
};
// Units total / workers each, the first total % workers of them one more.
struct Shares {
  int each, more;
  __device__ Shares(int total, int workers) : each((int)((uint32_t)total / (uint32_t)workers)), more(total - each * workers) {}
  __device__ int start(int w) const { return w * each + min(w, more); }
  __device__ int of(int unit) const {  // whose unit it is
    const int behind = unit - more * (each + 1);
    return behind < 0 ? (int)((uint32_t)unit / (uint32_t)(each + 1)) : more + (int)((uint32_t)behind / (uint32_t)each);
  }
};

// (by all 256 threads, a sequence in each; what they read of the one that u0 lies in goes along)
template <int COLS>
__device__ __forceinline__ Place find_place(const Attend4Args& a) {
  __shared__ int of_wave[2][4], found[6];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, batch = a.s.batch;
  const auto upto = [&](int n) {  // sums of lanes 0 .. this one
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(n, d);
      if (lane >= d) n = __builtin_elementwise_add_sat(n, o);
    }
    return n;
  };
  SeqRows s{};
  const auto units = [&](int b) {
    if (b >= batch) return 0;
    s = seq_rows(a.s, a.c.log_page, b);
    return seq_units<COLS>(a, s).units(a.c.heads);
  };
  // (sums stop at 2^31 - 1: with rows that descend, sequences share rows and the units are more than are counted)
  int all = 0;
  for (int base = 256; base < batch; base += 256) all = __builtin_elementwise_add_sat(all, units(base + tid));
  int n = units(tid), sum = upto(n);
  if (batch > 256) all = upto(all);
  if (lane == 63) {
    of_wave[0][wave] = sum;
    of_wave[1][wave] = all;
  }
  if (tid == 0) found[0] = batch;  // (unless what is read changes meanwhile)
  __syncthreads();
  Place p;
  p.total = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    p.total = __builtin_elementwise_add_sat(p.total, __builtin_elementwise_add_sat(of_wave[0][i], of_wave[1][i]));
  p.total = __builtin_amdgcn_readfirstlane(p.total);
  if (p.total > a.units) p.total = 0;  // nobody has a share (and the rows are reported)
  // an XCD's workgroups have neighbouring shares, and all XCDs have some
  p.workers = min(a.workers, p.total);
  const int each = (p.workers + 7) >> 3, i = (int)(blockIdx.x >> 3);
  p.w = (int)(blockIdx.x & 7) * each + i;
  if (i >= each || p.w >= p.workers) {  // without a share
    p.u0 = p.u1 = p.total;
    return p;
  }
  const Shares shares(p.total, p.workers);
  p.u0 = shares.start(p.w);
  p.u1 = shares.start(p.w + 1);
  int before = 0;
  for (int base = 0; base < batch; base += 256) {
    if (base) {
      __syncthreads();
      sum = upto(n = units(base + tid));
      if (lane == 63) of_wave[0][wave] = sum;
      __syncthreads();
    }
    int mine = before + sum - n;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      mine += w < wave ? of_wave[0][w] : 0;
      before += of_wave[0][w];
    }
    if (mine <= p.u0 && p.u0 < mine + n) {
      found[0] = base + tid;
      found[1] = mine;
      found[2] = s.row0;
      found[3] = s.n;
      found[4] = s.len;
    }
    if (before > p.u0) break;
  }
  __syncthreads();
  p.b = __builtin_amdgcn_readfirstlane(found[0]);
  p.before = __builtin_amdgcn_readfirstlane(found[1]);
  p.s.row0 = __builtin_amdgcn_readfirstlane(found[2]);
  p.s.n = __builtin_amdgcn_readfirstlane(found[3]);
  p.s.len = __builtin_amdgcn_readfirstlane(found[4]);
  return p;
}

__device__ __forceinline__ float max_of_columns(float v) {  // over the lanes l, l + 16, l + 32, l + 48
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const auto q = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

// Scale bytes with which a value may not be finite: 255, and above the quantiser's largest, what places hold that
// nothing was written to.  (A byte of ~w below 3 borrows.)
constexpr uint32_t kNotFinite = 253;
__device__ __forceinline__ uint32_t any_not_finite(uint32_t w) { return (~w - 0x03030303u) & w & 0x80808080u; }
// The word with these as 0.
__device__ __forceinline__ uint32_t only_finite(uint32_t w) {
  uint32_t o = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t b = w >> (8 * i) & 255u;
    o |= (b >= kNotFinite ? 0u : b) << (8 * i);
  }
  return o;
}

// A column's sums of one piece of the tokens, in powers of two of `m`.
__device__ __forceinline__ float lse_of(float m, float l) { return (m + __log2f(l)) * 0.6931471805599453f; }

template <int D>
struct Block {  // 32 tokens in a lane
  static constexpr int W = D / 32;  // words of keys per 16 tokens, and of values per 4
  uint32_t k[2][W], v[2 * W], vs[2];
  uint32_t ks[2];
};

// Block of 32 tokens, the `at`th of its page, of head `head` of all pages' heads.  (One base for
// the wave and a lane's own 32-bit offset: addresses take no registers but that.)
template <int D>
__device__ __forceinline__ void load_keys(Block<D>& x, const Cache4& c, int64_t head, int at, uint32_t l, uint32_t g,
                                          int one = -1) {  // one: of its halves alone, as the first
  constexpr uint32_t W = D / 32;
  const int64_t tok = (head << c.log_page) + at * 32 + max(one, 0) * 16;
  const uint8_t* k = c.k + (tok * D >> 1);
  const uint8_t* ks = c.ks + tok * W;
  const uint32_t kl = D == 64 ? (g >> 1) * 256 + l * 16 + (g & 1) * 8 : g * (2 * D) + l * 16;
  const uint32_t sl = l * W + (D == 64 ? g >> 1 : D == 128 ? g : 2 * g);
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    if (t && one >= 0) break;
    if constexpr (D == 64) {
      *reinterpret_cast<uint2*>(x.k[t]) = *reinterpret_cast<const uint2*>(k + t * (8 * D) + kl);
      x.ks[t] = (ks + t * (16 * W))[sl];
    } else if constexpr (D == 128) {
      *reinterpret_cast<uint4*>(x.k[t]) = *reinterpret_cast<const uint4*>(k + t * (8 * D) + kl);
      x.ks[t] = (ks + t * (16 * W))[sl];
    } else {
      *reinterpret_cast<uint4*>(x.k[t]) = *reinterpret_cast<const uint4*>(k + t * (8 * D) + kl);
      *reinterpret_cast<uint4*>(x.k[t] + 4) = *reinterpret_cast<const uint4*>(k + t * (8 * D) + 256 + kl);
      x.ks[t] = *reinterpret_cast<const uint16_t*>(ks + t * (16 * W) + sl);
    }
  }
}
template <int D>
__device__ __forceinline__ void load_values(Block<D>& x, const Cache4& c, int64_t head, int at, uint32_t l, uint32_t g) {
  const int64_t tok = (head << c.log_page) + at * 32;
  const uint8_t* v = c.v + (tok * D >> 1);
  const uint32_t vl = (l * 4 + g) * (D / 4), sl = l * D / 512 * 32 + g * 8;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const uint4 w = *reinterpret_cast<const uint4*>(v + i * 16 + vl);
    x.v[4 * i] = w.x;
    x.v[4 * i + 1] = w.y;
    x.v[4 * i + 2] = w.z;
    x.v[4 * i + 3] = w.w;
  }
  *reinterpret_cast<uint2*>(x.vs) = *reinterpret_cast<const uint2*>(c.vs + tok * (D / 32) + sl);
}

// Eight tokens' codes of the values 2 P and 2 P + 1 of a lane, as two operands: token j's
// are in byte P of its D / 32.
template <int D, int P>
__device__ __forceinline__ void values_pair(const uint32_t* v, const float* s, uint4& even, uint4& odd) {
  uint32_t u[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if constexpr (D == 64)
      u[j] = j & 1 ? mx4_pair<2 + (P & 1)>(v[j >> 1], s[j]) : mx4_pair<(P & 1)>(v[j >> 1], s[j]);
    else
      u[j] = mx4_pair<(P & 3)>(v[j * (D / 128) + P / 4], s[j]);
  }
  even = make_uint4(__builtin_amdgcn_perm(u[1], u[0], 0x05040100u), __builtin_amdgcn_perm(u[3], u[2], 0x05040100u),
                    __builtin_amdgcn_perm(u[5], u[4], 0x05040100u), __builtin_amdgcn_perm(u[7], u[6], 0x05040100u));
  odd = make_uint4(__builtin_amdgcn_perm(u[1], u[0], 0x07060302u), __builtin_amdgcn_perm(u[3], u[2], 0x07060302u),
                   __builtin_amdgcn_perm(u[5], u[4], 0x07060302u), __builtin_amdgcn_perm(u[7], u[6], 0x07060302u));
}

template <int D, int NC, int P>
__device__ __forceinline__ void add_values(f32x4_t (&o)[NC][D / 16], const uint32_t* v, const float* s, const bf16x8_t* p) {
  if constexpr (P < D / 32) {
    uint4 even, odd;
    values_pair<D, P>(v, s, even, odd);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      o[c][2 * P] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, even), p[c], o[c][2 * P], 0, 0, 0);
      o[c][2 * P + 1] =
          __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, odd), p[c], o[c][2 * P + 1], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);  // (all of it at once would spill)
    add_values<D, NC, P + 1>(o, v, s, p);
  }
}

// Operands of every other pair of values from number P on, into LDS.
template <int D, int P>
__device__ __forceinline__ void widen_values(unsigned char* to, const uint32_t* v, const float* s) {
  if constexpr (P < D / 32) {
    uint4 even, odd;
    values_pair<D, P>(v, s, even, odd);
    *reinterpret_cast<uint4*>(to + 2 * P * 1024) = even;
    *reinterpret_cast<uint4*>(to + (2 * P + 1) * 1024) = odd;
    widen_values<D, P + 2>(to, v, s);
  }
}

// Scores of tokens that a column does not see, of a block whose first one of this lane is t0.
template <int NC>
__device__ __forceinline__ void hide_tokens(f32x4_t (&sc)[2][NC], int t0, const int* pos, int window) {
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int from = window ? pos[c] - window : INT_MIN;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int tok = t0 + t * 16 + j;
        if (tok > pos[c] || tok <= from) sc[t][c][j] = kNegInf;
      }
  }
}

// From this size on (powers of two) a reference is `far`: it is a column's largest score as rounded to f32, and the
// exact product is off that by up to half a step of the score: 2^8 at 2^32, where a weight or its sum would overflow,
// or all weights underflow.  Below it that half step is at most 0.5, and the 6 ahead are not lost.
constexpr float kFar = 0x1p24f;

// A column's weights of 32 tokens, eight in a lane, to bf16.  far: whether the wave has a column with a far reference;
// such a column's scores are rounded as the reference was, so that the largest one's exponent is 0 to -8.
__device__ __forceinline__ uint4 weights(const f32x4_t s0, const f32x4_t s1, float scale, float off, bool far) {
  if (__builtin_expect(far, 0)) {
    const bool mine = fabsf(off) >= kFar;
    const auto power = [&](float x) {
#pragma clang fp contract(off)
      const float score = x * scale;
      return __builtin_amdgcn_exp2f(mine ? score + off : __builtin_fmaf(x, scale, off));
    };
    return make_uint4(bf16_pair(power(s0[0]), power(s0[1])), bf16_pair(power(s0[2]), power(s0[3])),
                      bf16_pair(power(s1[0]), power(s1[1])), bf16_pair(power(s1[2]), power(s1[3])));
  }
  const auto pair = [&](float x, float y) {
    return bf16_pair(__builtin_amdgcn_exp2f(__builtin_fmaf(x, scale, off)), __builtin_amdgcn_exp2f(__builtin_fmaf(y, scale, off)));
  };
  return make_uint4(pair(s0[0], s0[1]), pair(s0[2], s0[3]), pair(s1[0], s1[1]), pair(s1[2], s1[3]));
}
// Whether a column of the wave has no reference yet, or one that is too far behind: a weight of 2 or more has
// bit 14 set, and no other has (a NaN has too).
__device__ __forceinline__ bool behind(const uint4 p, float m) {
  return __ballot(((p.x | p.y | p.z | p.w) & 0x40004000u) != 0 || m == kNegInf) != 0;
}
// The reference that a column gets then, with the factor for what was summed up under the old one.
__device__ __forceinline__ float raise(const f32x4_t s0, const f32x4_t s1, float scale, float& m, float& off, bool& far) {
  const float big = scale * fmaxf(fmaxf(fmaxf(s0[0], s0[1]), fmaxf(s0[2], s0[3])), fmaxf(fmaxf(s1[0], s1[1]), fmaxf(s1[2], s1[3])));
  const float now = fmaxf(m, max_of_columns(big) + kAhead), shrink = now == m ? 1.f : __builtin_amdgcn_exp2f(m - now);
  m = now;
  off = now == kNegInf ? 0.f : -now;
  far |= __ballot(fabsf(off) >= kFar) != 0;
  return shrink;
}

// Columns that see a token of a block whose values are NaN (by its scale byte in vs) have NaN there: such a
// token counts 1 for the values of this lane, a token that a column sees 1 for it.
template <int NC, int NT>
__device__ __forceinline__ void mark_lost(f32x4_t (&o)[NC][NT], const uint32_t* vs, int t0, const int* pos, int window) {
  uint32_t na[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t pair = vs[j >> 1] >> (16 * (j & 1));
    na[j] = ((pair & 255u) >= kNotFinite ? 0x3f80u : 0u) | ((pair >> 8 & 255u) >= kNotFinite ? 0x3f800000u : 0u);
  }
  const bf16x8_t nan_at = __builtin_bit_cast(bf16x8_t, make_uint4(na[0], na[1], na[2], na[3]));
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    uint32_t se[4];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int tok = t0 + (j >> 2) * 16 + (j & 3);
      const bool sees = tok <= pos[c] && (!window || tok > pos[c] - window);
      const uint32_t one = sees ? 0x3f80u << (16 * (j & 1)) : 0u;
      se[j >> 1] = j & 1 ? se[j >> 1] | one : one;
    }
    const f32x4_t hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
        nan_at, __builtin_bit_cast(bf16x8_t, make_uint4(se[0], se[1], se[2], se[3])), f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[c][n][j] = hit[j] > 0.f ? NAN : o[c][n][j];
  }
}

}  // namespace

template <int D, int NC>
__global__ __launch_bounds__(256, attend_per_cu(D, NC)) void attend4_kernel(const Attend4Args a) {
  constexpr int COLS = 16 * NC, STEPS = D / 32, NT = D / 16, PITCH = D + 4;
  __shared__ __attribute__((aligned(16))) float part_o[4][16][PITCH];
  __shared__ float part_m[4][16], part_l[4][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l = lane & 15, g = lane >> 4;
  const Place place = find_place<COLS>(a);
  // (the records that belong to no share)
  if (tid == 0 && (int)blockIdx.x >= place.workers) a.shared()[blockIdx.x] = Shared{};
  if (place.u0 >= place.u1) return;
  const int w = place.w;
  const uint4 ones4 = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
  const bf16x8_t ones = __builtin_bit_cast(bf16x8_t, ones4);

  Shared shared{};  // the tile that begins here and goes on behind
  int u = place.u0, b = place.b, before = place.before;
  while (u < place.u1 && b < a.s.batch) {
    const SeqUnits q = seq_units<COLS>(a, b == place.b ? place.s : seq_rows(a.s, a.c.log_page, b));
    const int seq_total = q.units(a.c.heads);
    if (u - before >= seq_total) {
      before += seq_total;
      ++b;
      continue;
    }
    // the tile of columns and the units of it that are this workgroup's
    const int item = (u - before) / q.nb, start = u - before - item * q.nb;
    const int end = min(q.nb, start + place.u1 - u);
    const int h = item / q.ct, tile = item - h * q.ct;
    u += end - start;

    const int cols = (int)min((int64_t)COLS, (int64_t)q.s.n * a.group - (int64_t)tile * COLS);  // at least one
    const int r0 = tile * COLS / a.group, r1 = (tile * COLS + cols - 1) / a.group;  // rows of the sequence
    const int pos0 = q.s.len - q.s.n + r0, pos1 = q.s.len - q.s.n + r1;             // their tokens
    // this lane's columns
    bf16x8_t qv[NC][STEPS];
    int pos[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int col = tile * COLS + min(c * 16 + l, cols - 1), r = col / a.group, head = col - r * a.group;
      pos[c] = q.s.len - q.s.n + r;
      const uint16_t* at = a.q + (int64_t)(q.s.row0 + r) * a.q_row + (int64_t)(h * a.group + head) * a.q_head + g * (D / 4);
#pragma unroll
      for (int s = 0; s < STEPS; ++s) __builtin_memcpy(&qv[c][s], at + s * 8, 16);
    }
    f32x4_t o[NC][NT], sum[NC];
    float m[NC], off[NC];
    bool far = false;  // a column of the wave has a far reference
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int n = 0; n < NT; ++n) o[c][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      sum[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      m[c] = kNegInf;
      off[c] = 0.f;
    }

    // blocks of 32 tokens that any column of the tile sees
    int blk = (q.first + start) * 4, blk_end = min((q.first + end) * 4, (pos1 + 32) >> 5);
    if (a.window) blk = max(blk, max(0, pos0 - a.window + 1) >> 5);
    blk += wave;
    const int pages32 = a.c.log_page - 5, in_page = (1 << pages32) - 1;
    // (a page is asked for two blocks ahead, and held to bounds where it is used)
    const auto page_of = [&](int at) { return seq_page_raw(a.s, b, at >> pages32); };
    const auto head_of = [&](int page) { return (int64_t)page_in(a.s, a.c.n_pages, page) * a.c.heads + h; };
    const auto at_edge = [&](int at) {  // some column does not see all of its tokens
      return at * 32 + 31 > pos0 || (a.window && at * 32 <= pos1 - a.window);
    };
    Block<D> x;
    int next = 0;  // the next block's page
    bool lost = false;  // a block of values that is NaN where some column may not see it
    const int blk0 = blk;
    if (blk < blk_end) {
      const int page = page_of(blk);
      if (blk + 4 < blk_end) next = page_of(blk + 4);
      load_keys<D>(x, a.c, head_of(page), blk & in_page, l, g);
      load_values<D>(x, a.c, head_of(page), blk & in_page, l, g);
    }
    // A block's keys make room for the next one's as soon as the scores are there, its values when
    // they have been added: no second set of registers, and the other waves hide the loads.
    for (; blk < blk_end; blk += 4) {
      const bool more = blk + 4 < blk_end;
      const int64_t head = more ? head_of(next) : 0;
      if (blk + 8 < blk_end) next = page_of(blk + 8);
      f32x4_t sc[2][NC];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int c = 0; c < NC; ++c) sc[t][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        float s0, s1;
        if constexpr (D == 256) {
          s0 = mx4_scale(x.ks[t] & 255u);
          s1 = mx4_scale(x.ks[t] >> 8);
        } else {
          s0 = s1 = mx4_scale(x.ks[t]);
        }
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
          const bf16x8_t kv = __builtin_bit_cast(bf16x8_t, mx4_bf16x8(x.k[t][s], s < 4 ? s0 : s1));
#pragma unroll
          for (int c = 0; c < NC; ++c) sc[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kv, qv[c][s], sc[t][c], 0, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (more) load_keys<D>(x, a.c, head, (blk + 4) & in_page, l, g);
      if (at_edge(blk)) {
        hide_tokens<NC>(sc, blk * 32 + g * 4, pos, a.window);
        if (__ballot((any_not_finite(x.vs[0]) | any_not_finite(x.vs[1])) != 0)) {
          lost = true;  // (seen to behind the loop)
          x.vs[0] = only_finite(x.vs[0]);
          x.vs[1] = only_finite(x.vs[1]);
        }
      }
      bf16x8_t p[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        uint4 pw = weights(sc[0][c], sc[1][c], a.scale, off[c], far);
        if (behind(pw, m[c])) {
          const float shrink = raise(sc[0][c], sc[1][c], a.scale, m[c], off[c], far);
          sum[c] *= shrink;
#pragma unroll
          for (int n = 0; n < NT; ++n) o[c][n] *= shrink;
          pw = weights(sc[0][c], sc[1][c], a.scale, off[c], far);
        }
        p[c] = __builtin_bit_cast(bf16x8_t, pw);
        sum[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, p[c], sum[c], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
      float fs[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) fs[j] = mx4_scale(x.vs[j >> 2] >> (8 * (j & 3)) & 255u);
      add_values<D, NC, 0>(o, x.v, fs, p);
      if (more) load_values<D>(x, a.c, head, (blk + 4) & in_page, l, g);
    }
    if (lost) {
      for (int at = blk0; at < blk_end; at += 4)
        if (at_edge(at)) {
          load_values<D>(x, a.c, head_of(page_of(at)), at & in_page, l, g);
          mark_lost<NC, NT>(o, x.vs, at * 32 + g * 4, pos, a.window);
        }
    }

    // The four waves' sums, 16 columns at a time.
    const bool whole = start == 0 && end == q.nb;
    float* slot = a.parts + (int64_t)(2 * w + (start == 0)) * (COLS * (D + 2));
    if (start == 0 && !whole) {
      shared = Shared{min(Shares(place.total, place.workers).of(u - end + q.nb - 1), place.workers - 1), place.total, h, tile, cols, q.s.row0, q.s.len - q.s.n, 0};
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < NT; n += 4)
          *reinterpret_cast<float4*>(&part_o[wave][l][(4 * g + j) * NT + n]) =
              make_float4(o[c][n][j], o[c][n + 1][j], o[c][n + 2][j], o[c][n + 3][j]);
      if (g == 0) {
        part_m[wave][l] = m[c];
        part_l[wave][l] = sum[c][0];
      }
      __syncthreads();
      for (int e = tid; e < 16 * (D / 4); e += 256) {
        const int col = e / (D / 4), d = (e % (D / 4)) * 4;
        if (c * 16 + col >= cols) continue;
        const float top = fmaxf(fmaxf(part_m[0][col], part_m[1][col]), fmaxf(part_m[2][col], part_m[3][col]));
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        float ls = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float f = part_m[i][col] == top ? 1.f : __builtin_amdgcn_exp2f(part_m[i][col] - top);
          const float4 v = *reinterpret_cast<const float4*>(&part_o[i][col][d]);
          s = make_float4(s.x + f * v.x, s.y + f * v.y, s.z + f * v.z, s.w + f * v.w);
          ls += f * part_l[i][col];
        }
        if (!whole) {
          *reinterpret_cast<float4*>(slot + (c * 16 + col) * D + d) = s;
          if (d == 0) {
            slot[COLS * D + c * 16 + col] = top;
            slot[COLS * D + COLS + c * 16 + col] = ls;
          }
          continue;
        }
        const int at = tile * COLS + c * 16 + col, r = at / a.group, head = h * a.group + at - r * a.group;
        const int64_t row = q.s.row0 + r;
        const bool empty = q.s.len - q.s.n + r < 0;
        const float inv = 1.f / ls;
        store4(a.out, kBF16, row * a.o_row + head * a.o_head + d, 4,
               empty ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(s.x * inv, s.y * inv, s.z * inv, s.w * inv));
        if (a.lse && d == 0) a.lse[row * ((int64_t)a.c.heads * a.group) + head] = empty ? kNegInf : lse_of(top, ls);
      }
    }
  }
  if (tid == 0) a.shared()[w] = shared;
}

// Many columns: 128 of them in a workgroup, 32 in a wave.  64 tokens at a time are widened once
// for all four waves, each a quarter, into LDS, in the order of MFMA operands, while the 64 before are
// used; the codes of those behind are on their way meanwhile.  A wave keeps its columns to the
// end: nothing is joined in LDS.
template <int D>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void attend4_wide_kernel(const Attend4Args a) {
  constexpr int NC = 2, WCOLS = 16 * NC, COLS = 4 * WCOLS, STEPS = D / 32, NT = D / 16;
  constexpr int kKeys = 4 * STEPS * 1024, kBuffer = kKeys + 2 * NT * 1024;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * kBuffer];
  __shared__ int any_lost;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l = lane & 15, g = lane >> 4;
  const Place place = find_place<COLS>(a);
  // (the records that belong to no share)
  if (tid == 0 && (int)blockIdx.x >= place.workers) a.shared()[blockIdx.x] = Shared{};
  if (place.u0 >= place.u1) return;
  const int w = place.w;
  const uint4 ones4 = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
  const bf16x8_t ones = __builtin_bit_cast(bf16x8_t, ones4);

  Shared shared{};  // the tile that begins here and goes on behind
  int u = place.u0, b = place.b, before = place.before;
  while (u < place.u1 && b < a.s.batch) {
    const SeqUnits q = seq_units<COLS>(a, b == place.b ? place.s : seq_rows(a.s, a.c.log_page, b));
    const int seq_total = q.units(a.c.heads);
    if (u - before >= seq_total) {
      before += seq_total;
      ++b;
      continue;
    }
    const int item = (u - before) / q.nb, start = u - before - item * q.nb;
    const int end = min(q.nb, start + place.u1 - u);
    // (early and late tiles in turn: the late ones' rows see more tokens)
    const int h = item / q.ct, turn = item - h * q.ct, tile = turn & 1 ? q.ct - 1 - (turn >> 1) : turn >> 1;
    u += end - start;

    const int cols = (int)min((int64_t)COLS, (int64_t)q.s.n * a.group - (int64_t)tile * COLS);  // at least one
    const int lag = q.s.len - q.s.n;  // a row's token: lag + row
    const int pos0 = lag + tile * COLS / a.group, pos1 = lag + (tile * COLS + cols - 1) / a.group;
    // this wave's columns, and the tokens of its first and last one
    const int mine = min(max(cols - wave * WCOLS, 0), WCOLS), col0 = tile * COLS + wave * WCOLS;
    const int wpos0 = lag + col0 / a.group, wpos1 = mine ? lag + (col0 + mine - 1) / a.group : INT_MIN;
    bf16x8_t qv[NC][STEPS];
    int pos[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int col = min(col0 + c * 16 + l, tile * COLS + cols - 1), r = col / a.group, head = col - r * a.group;
      pos[c] = lag + r;
      const uint16_t* at = a.q + (int64_t)(q.s.row0 + r) * a.q_row + (int64_t)(h * a.group + head) * a.q_head + g * (D / 4);
#pragma unroll
      for (int s = 0; s < STEPS; ++s) __builtin_memcpy(&qv[c][s], at + s * 8, 16);
    }
    f32x4_t o[NC][NT], sum[NC];
    float m[NC], off[NC];
    bool far = false;  // a column of the wave has a far reference
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int n = 0; n < NT; ++n) o[c][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      sum[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      m[c] = kNegInf;
      off[c] = 0.f;
    }

    // steps of 64 tokens that any column of the tile sees; blocks of 32 that the sequence has
    int st = (q.first + start) * 2, st_end = min((q.first + end) * 2, (pos1 + 64) >> 6);
    if (a.window) st = max(st, max(0, pos0 - a.window + 1) >> 6);
    const int st0 = st, last_block = (q.s.len - 1) >> 5;
    // The first block that a column sees.  (The first step's other half lies before a window then and may have no page:
    // page 0 stands for it, and no column takes what is there.)
    const auto first_block = [&] { return max(st0 * 2, a.window ? max(0, pos0 - a.window + 1) >> 5 : 0); };
    const int pages32 = a.c.log_page - 5, in_page = (1 << pages32) - 1;
    const auto block_of = [&](int at) { return min(at * 2 + (wave >> 1), last_block); };  // this wave's half of a step
    // (a page is asked for a step ahead of its use, and held to bounds there)
    const auto page_of = [&](int at) { return seq_page_raw(a.s, b, block_of(at) >> pages32); };
    const auto head_of = [&](int page) { return (int64_t)page_in(a.s, a.c.n_pages, page) * a.c.heads + h; };
    const auto at_edge = [&](int at) {  // some column of the tile does not see all of its tokens
      return at * 64 + 63 > pos0 || (a.window && at * 64 <= pos1 - a.window);
    };
    Block<D> x;  // (of the keys, 16 tokens)
    const auto load = [&](int at, int page) {
      const int blk = block_of(at) & in_page;
      const int64_t head = head_of(page);
      load_keys<D>(x, a.c, head, blk, l, g, wave & 1);
      load_values<D>(x, a.c, head, blk, l, g);
    };
    // The codes at hand into a buffer.
    const auto widen = [&](unsigned char* to, int at) {
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        const float f = mx4_scale(D == 256 ? (s < 4 ? x.ks[0] & 255u : x.ks[0] >> 8) : x.ks[0]);
        *reinterpret_cast<uint4*>(to + (wave * STEPS + s) * 1024 + lane * 16) = mx4_bf16x8(x.k[0][s], f);
      }
      if (at_edge(at) && __ballot((any_not_finite(x.vs[0]) | any_not_finite(x.vs[1])) != 0)) {
        any_lost = 1;  // (seen to behind the loop)
        x.vs[0] = only_finite(x.vs[0]);
        x.vs[1] = only_finite(x.vs[1]);
      }
      float fs[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) fs[j] = mx4_scale(x.vs[j >> 2] >> (8 * (j & 3)) & 255u);
      // (the pairs of this wave's parity, all at the even ones' places in the words)
      uint32_t words[2 * STEPS];
#pragma unroll
      for (int i = 0; i < 2 * STEPS; ++i) words[i] = x.v[i] >> ((wave & 1) * 8);
      widen_values<D, 0>(to + kKeys + (wave >> 1) * (NT * 1024) + (wave & 1) * 2048 + lane * 16, words, fs);
    };
    __syncthreads();  // (the tile before has been read)
    if (tid == 0) any_lost = 0;
    if (st < st_end) {
      const int page = page_of(st);
      load(st, block_of(st) < first_block() ? 0 : page);
      int next = st + 1 < st_end ? page_of(st + 1) : 0;
      __syncthreads();
      widen(smem, st);
      if (st + 1 < st_end) {
        load(st + 1, next);
        if (st + 2 < st_end) next = page_of(st + 2);
      }
      __syncthreads();
      for (int i = 0; st < st_end; ++st, i ^= 1) {
        const unsigned char* from = smem + i * kBuffer + lane * 16;
        if (st + 1 < st_end) {
          widen(smem + (i ^ 1) * kBuffer, st + 1);
          if (st + 2 < st_end) load(st + 2, next);
          if (st + 3 < st_end) next = page_of(st + 3);
        }
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          const int t0 = st * 64 + half * 32;
          if (t0 > wpos1 || (a.window && t0 + 31 <= wpos0 - a.window)) continue;  // nothing that this wave's columns see
          f32x4_t sc[2][NC];
          const unsigned char* keys = from + half * (2 * STEPS * 1024);
          // (all of them requested at once: a wait between reads and MFMAs in turn costs each its latency)
          constexpr int AT_ONCE = STEPS < 8 ? 2 : 1;
#pragma unroll
          for (int tt = 0; tt < 2; tt += AT_ONCE) {
            bf16x8_t kb[AT_ONCE][STEPS];
#pragma unroll
            for (int t = 0; t < AT_ONCE; ++t)
#pragma unroll
              for (int s = 0; s < STEPS; ++s) kb[t][s] = *reinterpret_cast<const bf16x8_t*>(keys + ((tt + t) * STEPS + s) * 1024);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < AT_ONCE; ++t)
#pragma unroll
              for (int c = 0; c < NC; ++c) sc[tt + t][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
              for (int t = 0; t < AT_ONCE; ++t)
#pragma unroll
                for (int c = 0; c < NC; ++c)
                  sc[tt + t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb[t][s], qv[c][s], sc[tt + t][c], 0, 0, 0);
          }
          // (the first values are on their way while the weights are made)
          constexpr int EARLY = NT < 8 ? NT : 8;
          bf16x8_t vb[EARLY];
          const unsigned char* vals = from + kKeys + half * (NT * 1024);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int n = 0; n < EARLY; ++n) vb[n] = *reinterpret_cast<const bf16x8_t*>(vals + n * 1024);
          __builtin_amdgcn_sched_barrier(0);
          if (t0 + 31 > wpos0 || (a.window && t0 <= wpos1 - a.window)) {
            hide_tokens<NC>(sc, t0 + g * 4, pos, a.window);
          }
          bf16x8_t p[NC];
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            uint4 pw = weights(sc[0][c], sc[1][c], a.scale, off[c], far);
            if (behind(pw, m[c])) {
              const float shrink = raise(sc[0][c], sc[1][c], a.scale, m[c], off[c], far);
              sum[c] *= shrink;
#pragma unroll
              for (int n = 0; n < NT; ++n) o[c][n] *= shrink;
              pw = weights(sc[0][c], sc[1][c], a.scale, off[c], far);
            }
            p[c] = __builtin_bit_cast(bf16x8_t, pw);
            sum[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, p[c], sum[c], 0, 0, 0);
          }
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const bf16x8_t vv = n < EARLY ? vb[n < EARLY ? n : 0] : *reinterpret_cast<const bf16x8_t*>(vals + n * 1024);
#pragma unroll
            for (int c = 0; c < NC; ++c) o[c][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, p[c], o[c][n], 0, 0, 0);
          }
        }
        __syncthreads();
      }
      if (any_lost) {
        for (int at = st0 * 2; at < st_end * 2 && at <= last_block; ++at)
          if (at_edge(at >> 1)) {
            load_values<D>(x, a.c, head_of(at < first_block() ? 0 : seq_page_raw(a.s, b, at >> pages32)), at & in_page, l, g);
            mark_lost<NC, NT>(o, x.vs, at * 32 + g * 4, pos, a.window);
          }
      }
    }

    const bool whole = start == 0 && end == q.nb;
    float* slot = a.parts + (int64_t)(2 * w + (start == 0)) * (COLS * (D + 2));
    if (start == 0 && !whole)
      shared = Shared{min(Shares(place.total, place.workers).of(u - end + q.nb - 1), place.workers - 1), place.total, h, tile, cols, q.s.row0, lag, 0};
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int col = wave * WCOLS + c * 16 + l;
      if (col >= cols) continue;
      const int at = tile * COLS + col, r = at / a.group, head = h * a.group + at - r * a.group;
      const int64_t row = q.s.row0 + r;
      const bool empty = lag + r < 0;
      const float inv = 1.f / sum[c][0];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int d = (4 * g + j) * NT;
#pragma unroll
        for (int n = 0; n < NT; n += 4) {
          const float4 v = make_float4(o[c][n][j], o[c][n + 1][j], o[c][n + 2][j], o[c][n + 3][j]);
          if (whole)
            store4(a.out, kBF16, row * a.o_row + head * a.o_head + d + n, 4,
                   empty ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
          else
            *reinterpret_cast<float4*>(slot + col * D + d + n) = v;
        }
      }
      if (g == 0) {
        if (!whole) {
          slot[COLS * D + col] = m[c];
          slot[COLS * D + COLS + col] = sum[c][0];
        } else if (a.lse) {
          a.lse[row * ((int64_t)a.c.heads * a.group) + head] = empty ? kNegInf : lse_of(m[c], sum[c][0]);
        }
      }
    }
  }
  if (tid == 0) a.shared()[w] = shared;
}

// The parts of a tile, joined: workgroup (w, y) does that for the tile that begins in w's share and
// goes on behind it, if there is one.  A lane has four values of a column, a wave 256 / D
// columns.  SPLIT (few columns, perhaps many parts): the eight waves have the same columns and every eighth
// part each, and are joined in LDS; else each has columns of its own.
template <int D, int COLS, bool SPLIT>
__global__ __launch_bounds__(512) void attend4_join_kernel(const Attend4Args a) {
  constexpr int SLOT = COLS * (D + 2), LANES = D / 4, PER = 64 / LANES, STEP = SPLIT ? 8 : 1;
  __shared__ float4 part_v[8][64];
  __shared__ float part_m[8][64], part_l[8][64];
  const int w = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Shared t = a.shared()[w];
  const int n = t.last - w + 1;  // workgroups that have a part
  const int first = (SPLIT ? blockIdx.y : blockIdx.y * 8 + wave) * PER;
  if (n <= 1 || first >= t.cols) return;
  const int col = first + lane / LANES, d = lane % LANES * 4;
  const bool real = col < t.cols;
  const float* at = a.parts + (int64_t)(2 * w) * SLOT;
  float top = kNegInf, ls = 0.f;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  const auto add = [&](float m, float l, const float4 v) {
    const float now = fmaxf(top, m);
    const float f0 = top == now ? 1.f : __builtin_amdgcn_exp2f(top - now), f1 = m == now ? 1.f : __builtin_amdgcn_exp2f(m - now);
    s = make_float4(s.x * f0 + v.x * f1, s.y * f0 + v.y * f1, s.z * f0 + v.z * f1, s.w * f0 + v.w * f1);
    ls = ls * f0 + l * f1;
    top = now;
  };
  for (int i = SPLIT ? wave : 0; i < n; i += 4 * STEP) {
    float m[4], l[4];
    float4 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int p = i + STEP * j;
      m[j] = kNegInf;
      l[j] = 0.f;
      v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (real && p < n) {
        const float* slot = at + (int64_t)(p ? 2 * p : 1) * SLOT;
        m[j] = slot[COLS * D + col];
        l[j] = slot[COLS * D + COLS + col];
        v[j] = *reinterpret_cast<const float4*>(slot + col * D + d);
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) add(m[j], l[j], v[j]);
  }
  if constexpr (SPLIT) {
    part_v[wave][lane] = s;
    part_m[wave][lane] = top;
    part_l[wave][lane] = ls;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) add(part_m[i][lane], part_l[i][lane], part_v[i][lane]);
  }
  if (!real) return;
  const int c = t.tile * COLS + col, r = c / a.group, head = t.head * a.group + c - r * a.group;
  const int64_t row = t.row0 + r;
  const bool empty = t.pos0 + r < 0;
  const float inv = 1.f / ls;
  store4(a.out, kBF16, row * a.o_row + head * a.o_head + d, 4,
         empty ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(s.x * inv, s.y * inv, s.z * inv, s.w * inv));
  if (a.lse && d == 0) a.lse[row * ((int64_t)a.c.heads * a.group) + head] = empty ? kNegInf : lse_of(top, ls);
}

template <int D, int NC>
static hipError_t attend_launch(const Attend4Args& a, hipStream_t s) {
  constexpr bool WIDE = NC == kAttendWide;
  if constexpr (WIDE) {
    attend4_wide_kernel<D><<<a.workers, 256, 0, s>>>(a);
  } else {
    attend4_kernel<D, NC><<<a.workers, 256, 0, s>>>(a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // (a tile's columns, as many as there can be)
  const int64_t cols = a.s.rows ? 16 * NC : std::min<int64_t>(16 * NC, (int64_t)a.s.n * a.group);
  const int64_t waves = (cols * D + 255) / 256;
  attend4_join_kernel<D, 16 * NC, !WIDE><<<dim3(a.workers, (unsigned)(WIDE ? (waves + 7) / 8 : waves)), 512, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_attend4(const Attend4Args& a, hipStream_t s) {
  switch (a.c.d * 8 + (a.nc == kAttendWide ? 3 : a.nc)) {
    case 64 * 8 + 1: return attend_launch<64, 1>(a, s);
    case 64 * 8 + 2: return attend_launch<64, 2>(a, s);
    case 64 * 8 + 3: return attend_launch<64, kAttendWide>(a, s);
    case 128 * 8 + 1: return attend_launch<128, 1>(a, s);
    case 128 * 8 + 2: return attend_launch<128, 2>(a, s);
    case 128 * 8 + 3: return attend_launch<128, kAttendWide>(a, s);
    case 256 * 8 + 1: return attend_launch<256, 1>(a, s);
    case 256 * 8 + 2: return attend_launch<256, 2>(a, s);
    default: return attend_launch<256, kAttendWide>(a, s);
  }
}

}  // namespace aep
