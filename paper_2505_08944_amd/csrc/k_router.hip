// Routing by scores: softmax or sigmoid scores, a bias for the choice, expert
// groups, top-k, weights from the scores of the chosen (the rule is stated at
// aep_router in aep.h).
//
// A token takes 16 lanes of a wave (32 above 256 experts), each holding up to
// 16 of its experts.  Experts are compared as one f64 per expert: the f32 choice
// (or logit) in its upper bits, the expert's id in the 29 that an f32 leaves
// free, so that a single maximum orders by choice, then by id.  Every lane
// sorts its keys with a network of maxima and minima; a selection round is then
// a maximum over the lanes' heads by DPP, and the winner's lane moves up.
//
// The rule compares choices in binary64, as a score plus a bias of like size
// has neighbours that binary32 cannot tell apart, and the same logits must give
// the same experts on every rank.  Where all neighbours in the order, and the
// last kept and first dropped group, are further apart than f32's errors, f32 has
// given the rule's answer.  Where they are not (one token in a few hundred), the
// choices in question, one per lane, or the groups, are compared again in f64.
// Logits without a bias are compared as they are, exactly.
//
// What bounds it: 8192 tokens of 256 experts in 8 groups, sigmoid and bias, 13.3
// us (8.9 MB: 1.7 us at the rate of a large copy): 1600 vector instructions per
// wave of four tokens, two waves per SIMD; a further 8192 tokens take 5.4.  (A
// wave per token, all of it in f64: 34 us.)  64 tokens: 7.4 us, one wave's chain
// of loads, sort, rounds and f64 weights; 1.8 more where a token's choices have
// to be compared in f64.
#include <float.h>
#include <limits.h>

#include <type_traits>
#include <utility>

#include "aep_internal.h"
#include "route_token_id.h"

namespace aep {

// ------------------------------------------------------- lanes of one token
// Lane l's value from lane l ^ 1, l ^ 2 (within four), 7 - l (within eight),
// 15 - l (within 16): after a reduction over the steps before, each completes
// the next one.  Step 4 (two rows of 16) goes through LDS permutes.
template <int STEP>
__device__ __forceinline__ int partner(int v) {
  if constexpr (STEP == 4) return __shfl_xor(v, 16);
  constexpr int ctrl = STEP == 0 ? 0xB1 : STEP == 1 ? 0x4E : STEP == 2 ? 0x141 /* row_half_mirror */ : 0x140 /* row_mirror */;
  return __builtin_amdgcn_update_dpp(0, v, ctrl, 0xF, 0xF, true);
}
template <int STEP>
__device__ __forceinline__ float partner(float v) {
  return __int_as_float(partner<STEP>(__float_as_int(v)));
}
template <int STEP>
__device__ __forceinline__ double partner(double v) {
  return __hiloint2double(partner<STEP>(__double2hiint(v)), partner<STEP>(__double2loint(v)));
}
template <int LANES, typename T, typename F>
__device__ __forceinline__ T reduce(T v, F f) {
  v = f(v, partner<0>(v));
  v = f(v, partner<1>(v));
  v = f(v, partner<2>(v));
  v = f(v, partner<3>(v));
  if constexpr (LANES == 32) v = f(v, partner<4>(v));
  return v;
}
__device__ __forceinline__ double max64(double a, double b) { return __builtin_fmax(a, b); }
template <int LANES>
__device__ __forceinline__ double reduce_max(double v) {
  return reduce<LANES>(v, [](double a, double b) { return max64(a, b); });
}

// -------------------------------------------------------------------- keys
// f32 value and id (below 512) in one f64: larger value first, equal: lower id.
constexpr int kIdMask = 511;
__device__ __forceinline__ double make_key(float v, int id) {
  const double d = (double)(v + 0.f);  // -0 becomes +0
  const int lo = __double2loint(d), hi = __double2hiint(d);
  return __hiloint2double(hi, lo | (hi < 0 ? id : kIdMask - id));
}
__device__ __forceinline__ int key_id(double k) {
  const int lo = __double2loint(k) & kIdMask;
  return __double2hiint(k) < 0 ? lo : kIdMask - lo;
}
// Below every f32: masked experts, by id, and then those that may not be picked.
__device__ __forceinline__ double masked_key(int id) { return __hiloint2double((int)0xFE000000u, id); }
__device__ __forceinline__ double never_key() { return -DBL_MAX; }
__device__ __forceinline__ bool is_live(double k) { return k > -1e100; }
// A key's value (its id is below half a step); -inf for those two.
__device__ __forceinline__ float key_value(double k) { return (float)k; }
static_assert(kMaxScoredExperts <= kIdMask + 1, "an id in kIdMask");

// Neighbours a >= b that are further apart than both errors: slack for the
// scores' part of them, and 2^-23 of the values for the additions, which are off
// by half a step, 2^-24, of each result.  A sigmoid is off by less than 2^-22 (the
// reciprocal 2^-23 and 1 + e^-x 2^-24 of it; e^-x 2^-23, and 2^-24 |x| for its
// argument, of s (1 - s)), a softmax score by 2^-20 of the largest one (e^x and
// their sum 2^-22 each, the reciprocal 2^-23); two scores twice
// that, two sums of two four times (of softmax scores, whose sum is at most 1,
// twice).
__device__ __forceinline__ bool apart(float a, float b, float slack) {
  // (-inf, a masked one, is apart from every other)
  return b == -__builtin_inff() || a - b > slack + 0x1p-23f * (fabsf(a) + fabsf(b));
}

// e^x for x <= 0 to 2^-22: the hardware's 2^x on the rounded x log2(e),
// corrected for what the rounding lost.  0 below -200, -inf included.
__device__ __forceinline__ float exp_neg(float x) {
  x = fmaxf(x, -200.f);
  const float t = x * 1.44269504f;
  const float lost = __builtin_fmaf(x, 1.44269504f, -t) + x * 1.925963033e-8f;
  const float e = __builtin_amdgcn_exp2f(t);
  return __builtin_fmaf(e, lost * 0.693147181f, e);
}
// 1 / (1 + e^-x); its error is stated at apart().
__device__ __forceinline__ float sigmoid32(float x) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * -1.44269504f));
}
__device__ __forceinline__ double sigmoid64(double x) { return 1.0 / (1.0 + exp(-x)); }

// Sorts a lane's N keys, largest first: odd-even merge sort (Batcher 1968), its
// comparators listed at compile time so that every key stays in a register.
template <int N>
struct SortNet {
  int n = 0, a[64] = {}, b[64] = {};
  constexpr SortNet() {
    for (int p = 1; p < N; p *= 2)
      for (int q = p; q >= 1; q /= 2)
        for (int j = q % p; j <= N - 1 - q; j += 2 * q)
          for (int i = 0; i < q; ++i)
            if (i + j + q < N && (i + j) / (p * 2) == (i + j + q) / (p * 2)) {
              a[n] = i + j;
              b[n] = i + j + q;
              ++n;
            }
  }
};
template <int N, size_t... I>
__device__ __forceinline__ void sort_steps(double (&k)[N], std::index_sequence<I...>) {
  constexpr SortNet<N> net;
  auto step = [](double& x, double& y) {
    const double hi = max64(x, y);
    y = __builtin_fmin(x, y);
    x = hi;
  };
  (step(k[net.a[I]], k[net.b[I]]), ...);
}
template <int N>
__device__ __forceinline__ void sort_keys(double (&k)[N]) {
  constexpr SortNet<N> net;
  sort_steps<N>(k, std::make_index_sequence<net.n>{});
}
// The largest L of a lane's N keys, sorted: of 16, two sorted eights whose
// larger halves (one list against the other reversed) are sorted once more.
template <int N, int L>
__device__ __forceinline__ void best_keys(const double (&k)[N], double (&out)[L]) {
  if constexpr (N == L) {
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = k[i];
    sort_keys<N>(out);
  } else {
    static_assert(N == 2 * L, "two lists");
    double a[L], b[L];
#pragma unroll
    for (int i = 0; i < L; ++i) {
      a[i] = k[i];
      b[i] = k[L + i];
    }
    sort_keys<L>(a);
    sort_keys<L>(b);
#pragma unroll
    for (int i = 0; i < L; ++i) out[i] = max64(a[i], b[L - 1 - i]);
    // a bitonic sequence: log2 L rounds of halves
#pragma unroll
    for (int h = L / 2; h >= 1; h /= 2)
#pragma unroll
      for (int i = 0; i < L; ++i)
        if (!(i & h)) {
          const double hi = max64(out[i], out[i + h]);
          out[i + h] = __builtin_fmin(out[i], out[i + h]);
          out[i] = hi;
        }
  }
}
// The largest of the lanes' sorted lists; its lane moves up, to `end` at last:
// never_key() where the list held all of the lane's experts, unknown_key(),
// which is then the largest, where it did not.
__device__ __forceinline__ double unknown_key() { return DBL_MAX; }
template <int LANES, int N>
__device__ __forceinline__ double take_best(double (&k)[N], double end) {
  const double w = reduce_max<LANES>(k[0]);
  const bool mine = k[0] == w;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    double a = k[i], b = i + 1 < N ? k[i + 1] : end;
    asm("" : "+v"(a), "+v"(b));  // a choice of two values: not of two places, which would index registers
    k[i] = mine ? b : a;
  }
  return w;
}

// The larger value, equal: the lower id; id INT_MAX: none.
__device__ __forceinline__ void better(double& v, int& e, double ov, int oe) {
  if (oe != INT_MAX && (e == INT_MAX || ov > v || (ov == v && oe < e))) {
    v = ov;
    e = oe;
  }
}
template <int LANES>
__device__ __forceinline__ void best_of(double& v, int& e) {
  better(v, e, partner<0>(v), partner<0>(e));
  better(v, e, partner<1>(v), partner<1>(e));
  better(v, e, partner<2>(v), partner<2>(e));
  better(v, e, partner<3>(v), partner<3>(e));
  if constexpr (LANES == 32) better(v, e, partner<4>(v), partner<4>(e));
}

// Calls f with the value and id of each of the token's other lanes.
template <typename F, size_t... D>
__device__ __forceinline__ void others_in_row(double v, int e, F f, std::index_sequence<D...>) {
  auto from = [](int x, auto d) {  // row_ror: a rotation of the 16 lanes
    return __builtin_amdgcn_update_dpp(0, x, 0x121 + d(), 0xF, 0xF, true);
  };
  (f(__hiloint2double(from(__double2hiint(v), std::integral_constant<int, D>{}),
                      from(__double2loint(v), std::integral_constant<int, D>{})),
     from(e, std::integral_constant<int, D>{})),
   ...);
}
template <int LANES, typename F>
__device__ __forceinline__ void others(double v, int e, F f) {
  others_in_row(v, e, f, std::make_index_sequence<15>{});
  if constexpr (LANES == 32) {
    const double w = partner<4>(v);
    const int o = partner<4>(e);
    f(w, o);
    others_in_row(w, o, f, std::make_index_sequence<15>{});
  }
}

// What a token's lanes share in LDS where experts have groups: a value per
// expert.  Its lanes are in one wave: ordering the wave's accesses is enough.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ------------------------------------------------------------------ groups
// How a token's lanes hold its experts.  Without groups, or with groups that
// do not fit whole lanes, lane g holds g, g + LANES, ...; the groups' worths are
// then found through LDS.  Where LANES / n_groups lanes hold a group each (16, 8,
// 4 or 2 groups, and 32 above 256 experts), lane g holds a run of E / LANES experts:
// a group's worth is a reduction over its lanes, and dropping a group is
// dropping its lanes' heads.
enum { kNoGroups = 0, kGroupLanes = 1, kGroupsInLds = 2 };

// The two largest of what has been added (-inf: nothing).
template <typename T>
struct Two {
  T a, b;
  __device__ __forceinline__ void add(T x) {
    b = x > a ? a : (x > b ? x : b);
    a = x > a ? x : a;
  }
  template <int STEP>
  __device__ __forceinline__ void join() {
    const T oa = partner<STEP>(a), ob = partner<STEP>(b);
    const T lo = oa > a ? a : oa, nb = ob > b ? ob : b;
    a = oa > a ? oa : a;
    b = lo > nb ? lo : nb;
  }
  // over `share` lanes, a power of two below LANES
  __device__ __forceinline__ void join_lanes(int share) {
    if (share > 1) join<0>();
    if (share > 2) join<1>();
    if (share > 4) join<2>();
    if (share > 8) join<3>();
  }
  // (f32: a sum past its range is its largest value, which is apart() from smaller
  // ones and never from another such sum; an infinity would be a masked group's
  // worth or, with an id in its bits, no number)
  __device__ __forceinline__ T worth(int group_top) const {
    T sum = a + b;
    if constexpr (sizeof(T) == 4) sum = fminf(fmaxf(sum, -FLT_MAX), FLT_MAX);
    return group_top > 1 && b != -(T)__builtin_inff() ? sum : a;
  }
};

// The top_groups best of Q groups per lane, group lead + q * step worth[q] (-inf:
// all masked), as a mask.  certain: no other f32 rounding would have kept
// others (slack < 0: the values are exact).
template <int LANES, int Q, typename T>
__device__ __forceinline__ uint64_t pick_groups(const T (&worth)[Q], int lead, int step, const RouterArgs& r, float slack,
                                                bool& certain) {
  const T none = -(T)__builtin_inff();
  uint64_t kept = 0;
  certain = true;
  if constexpr (sizeof(T) == 4) {
    double key[Q];
    float last = 0.f;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int gr = lead + q * step;
      key[q] = gr >= r.n_groups ? never_key() : worth[q] == none ? masked_key(gr) : make_key(worth[q], gr);
    }
    for (int j = 0; j <= r.top_groups; ++j) {
      double k = key[0];
#pragma unroll
      for (int q = 1; q < Q; ++q) k = max64(k, key[q]);
      k = reduce_max<LANES>(k);
      if (j == r.top_groups) {
        certain = slack < 0.f || apart(last, key_value(k), slack);
        break;
      }
      last = key_value(k);
      kept |= 1ull << key_id(k);
#pragma unroll
      for (int q = 0; q < Q; ++q) key[q] = key[q] == k ? never_key() : key[q];
    }
  } else {
    for (int j = 0; j < r.top_groups; ++j) {
      double v = none;
      int id = INT_MAX;
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const int gr = lead + q * step;
        if (gr < r.n_groups && !((kept >> gr) & 1)) better(v, id, (double)worth[q], gr);
      }
      best_of<LANES>(v, id);
      kept |= 1ull << id;
    }
  }
  return kept;
}

// The same from the experts' values in LDS; the lanes share the groups, 1 << shift
// lanes each where groups are few.
template <int LANES, typename T>
__device__ __forceinline__ uint64_t pick_groups_lds(const T* __restrict__ val, const RouterArgs& r, int g, float slack,
                                                    bool& certain) {
  const int per = r.per, shift = LANES == 32 ? r.share32 : r.share16, share = 1 << shift;
  const int sub = g & (share - 1), lead = g >> shift, step = LANES >> shift;
  const T none = -(T)__builtin_inff();
  T worth[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int gr = lead + q * step;
    Two<T> two{none, none};
    if (gr < r.n_groups) {
      // four at a time, so that their reads are in flight together
      for (int i = sub; i < per; i += 4 * share) {
        T x[4];
#pragma unroll
        for (int z = 0; z < 4; ++z) x[z] = val[gr * per + min(i + z * share, per - 1)];
#pragma unroll
        for (int z = 0; z < 4; ++z) two.add(i + z * share < per ? x[z] : none);
      }
    }
    two.join_lanes(share);
    worth[q] = two.worth(r.group_top);
    if (step * (q + 1) >= r.n_groups) {
#pragma unroll
      for (int z = q + 1; z < 4; ++z) worth[z] = none;
      break;
    }
  }
  return pick_groups<LANES, 4>(worth, lead, step, r, slack, certain);
}

// The experts of lane g: id(i), i < EPL, if has(i).
template <int LANES, int GM>
struct Held {
  int first, n, E;
  __device__ __forceinline__ Held(int g, int E) : first(GM == kGroupLanes ? g * (E / LANES) : g), n(E / LANES), E(E) {}
  __device__ __forceinline__ int id(int i) const { return GM == kGroupLanes ? first + i : first + i * LANES; }
  __device__ __forceinline__ bool has(int i) const { return GM == kGroupLanes ? i < n : id(i) < E; }
};

// This lane's values of a row (anything where there is none).  Runs are read in
// 16 bytes where their alignment allows (r.vec4): a load of lanes that are apart
// takes a cycle per lane.
template <int EPL, int LANES, int GM>
__device__ __forceinline__ void held_values(float (&v)[EPL], const float* __restrict__ row, const Held<LANES, GM>& held,
                                            const RouterArgs& r) {
  if (GM == kGroupLanes && r.vec4) {
#pragma unroll
    for (int i = 0; i < EPL; i += 4) {
      const float4 q = *reinterpret_cast<const float4*>(row + min(held.id(i), r.E - 4));
      v[i] = q.x;
      v[i + 1] = q.y;
      v[i + 2] = q.z;
      v[i + 3] = q.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) v[i] = row[min(held.id(i), r.E - 1)];
  }
}

// The groups that stay, where LANES / n_groups lanes hold a group each, from the
// two largest of each lane's values (-inf: masked or none), which become the
// group's.
template <int EPL, typename T>
__device__ __forceinline__ Two<T> two_of(const T (&c)[EPL]) {
  Two<T> two{-(T)__builtin_inff(), -(T)__builtin_inff()};
#pragma unroll
  for (int i = 0; i < EPL; ++i) two.add(c[i]);
  return two;
}
template <int LANES, typename T>
__device__ __forceinline__ uint64_t pick_group_lanes(Two<T>& two, const RouterArgs& r, int g, float slack, bool& certain) {
  const int shift = LANES == 32 ? r.share32 : r.share16;
  two.join_lanes(1 << shift);
  const T worth[1] = {two.worth(r.group_top)};
  return pick_groups<LANES, 1>(worth, g >> shift, LANES, r, slack, certain);
}

// The whole selection in f64, for a token with more choices too close to each
// other than it has lanes: lane j gets slot j's expert.  All of its lanes call it.
template <int EPL, int LANES, int GM>
__device__ __noinline__ int select_exact(const float* __restrict__ l, const float* __restrict__ bias, RouterArgs r, int g,
                                         double* __restrict__ val) {
  const double none = -__builtin_inf();
  const Held<LANES, GM> held{g, r.E};
  // without a bias experts are picked by their logits, and so are groups by their best one
  const bool by_logit = !bias && r.group_top == 1;
  double top = none, total = 0.0;
  if (!r.sigmoid && !by_logit) {
    for (int i = 0; i < EPL; ++i) {
      const int e = held.id(i);
      if (held.has(i) && __builtin_isfinite(l[e])) top = max64(top, (double)l[e]);
    }
    top = reduce_max<LANES>(top);
    for (int i = 0; i < EPL; ++i) {
      const int e = held.id(i);
      if (held.has(i) && __builtin_isfinite(l[e])) total += exp((double)l[e] - top);
    }
    total = reduce<LANES>(total, [](double a, double b) { return a + b; });
  }
  double c[EPL];
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int e = held.id(i);
    c[i] = none;
    if (held.has(i) && __builtin_isfinite(l[e])) {
      const double x = (double)l[e];
      c[i] = by_logit ? x : r.sigmoid ? sigmoid64(x) : exp(x - top) / total;
      if (bias) c[i] += (double)bias[e];
      if (!__builtin_isfinite(c[i])) c[i] = none;
    }
    if (GM == kGroupsInLds && held.has(i)) val[e] = c[i];
  }
  uint64_t kept = ~0ull;
  bool certain;
  if constexpr (GM == kGroupsInLds) {
    wave_fence();
    kept = pick_groups_lds<LANES, double>(val, r, g, -1.f, certain);
  }
  if constexpr (GM == kGroupLanes) {
    Two<double> two = two_of<EPL>(c);
    kept = pick_group_lanes<LANES>(two, r, g, -1.f, certain);
  }
  unsigned avail = 0;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int e = held.id(i);
    if (held.has(i) && ((kept >> (GM == kNoGroups ? 0 : e / r.per)) & 1)) avail |= 1u << i;
    if (!bias && c[i] != none) c[i] = (double)l[e];
  }
  int mine = 0;
  for (int j = 0; j < r.k; ++j) {
    double v = none;
    int id = INT_MAX;
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if ((avail >> i) & 1) better(v, id, c[i], held.id(i));
    best_of<LANES>(v, id);
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (held.id(i) == id) avail &= ~(1u << i);
    if (g == j) mine = id;
  }
  return mine;
}

// What the selection compares: the logits alone, or scores as well (choices with
// a bias, sums of two scores as groups' worths).
enum { kByLogit = 0, kBySoftmax = 1, kBySigmoid = 2 };

// Routes token t on its LANES lanes: lane j < k gets slot j's expert and weight.
// val: the token's LDS row (of E values; unused without groups).  bad: a value
// to be reported was seen by this lane.
template <int EPL, int LANES, int BY, int GM>
__device__ __forceinline__ void route_scored(const float* __restrict__ logits, int64_t ld,
                                             const float* __restrict__ bias, const RouterArgs& r, int64_t t, int g,
                                             double* __restrict__ val, int& my_e, float& my_w, bool& bad) {
  const float* __restrict__ l = logits + t * ld;
  const float none = -__builtin_inff();
  const Held<LANES, GM> held{g, r.E};
  float x[EPL], b[EPL];
  held_values<EPL>(x, l, held, r);
  if (BY != kByLogit && bias) {
    held_values<EPL>(b, bias, held, r);
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) b[i] = 0.f;
  }
  bad = false;
  float top = none;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    // a difference of a finite value with itself is 0, of any other NaN
    const bool live = x[i] - x[i] == 0.f;
    bad |= !live && x[i] != none && held.has(i);
    x[i] = live && held.has(i) ? x[i] : none;
  }
  const bool softmax = BY == kBySoftmax || (BY == kByLogit && !r.sigmoid);
  float total = 1.f;
  double sum_exp = 1.0;
  if (softmax) {
#pragma unroll
    for (int i = 0; i < EPL; ++i) top = fmaxf(top, x[i]);
    top = reduce<LANES>(top, [](float a, float b) { return fmaxf(a, b); });
    top = top == none ? 0.f : top;  // every expert masked
    if (BY == kBySoftmax || !r.renorm) {
      // (weights that are not renormalised are divided by it: added up in f64, from f32
      // exponentials of 2^-22 each, whose mean is far closer: 777 tokens' weights are
      // off by 2.7e-8 rms of 2.5e-8 that rounding them to f32 leaves.  f64 exponentials of
      // every expert would take some 30 instructions each; weights that are
      // renormalised use them, for the chosen experts)
      double z = 0.0;
#pragma unroll
      for (int i = 0; i < EPL; ++i) z += (double)exp_neg(x[i] - top);
      sum_exp = reduce<LANES>(z, [](double a, double b) { return a + b; });
      total = (float)sum_exp;
    }
  }
  // choices, or logits; with groups, what an expert is worth to its group
  const float inv = BY == kBySoftmax ? __builtin_amdgcn_rcpf(total) : 1.f;
  float* __restrict__ val32 = reinterpret_cast<float*>(val);
  double key[EPL];
  float val_of[EPL];
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int e = held.id(i);
    float c = x[i];
    if constexpr (BY == kBySoftmax) c = exp_neg(x[i] - top) * inv + b[i];
    if constexpr (BY == kBySigmoid) c = sigmoid32(x[i]) + b[i];
    const bool off = BY != kByLogit && c - c != 0.f && x[i] != none;  // a bias that is not finite
    bad |= off;
    c = x[i] == none || off ? none : c;
    val_of[i] = c;
    if (GM == kGroupsInLds && held.has(i)) val32[e] = c;
    const float by = BY == kByLogit || bias ? c : x[i];
    // (without runs, ids past E come behind every expert: none is picked)
    const double off_key = GM != kGroupLanes || held.has(i) ? masked_key(e) : never_key();
    key[i] = c == none ? off_key : make_key(by, e);
  }
  // (the largest softmax score is inv; the sum of a group's two may be 1)
  const float slack = BY == kBySoftmax ? 0x1p-18f * inv : 0x1p-21f;
  const float group_slack = BY == kByLogit ? -1.f : BY == kBySoftmax ? 0x1p-18f : 0x1p-20f;
  // softmax in f64, where it is needed
  auto total64 = [&] {
    double z = 0.0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) z += x[i] == none ? 0.0 : exp((double)x[i] - (double)top);
    return reduce<LANES>(z, [](double a, double b) { return a + b; });
  };
  auto choice64 = [&](float v, float bv, double z) {
    return (BY == kBySigmoid ? sigmoid64((double)v) : exp((double)v - (double)top) / z) + (double)bv;
  };
  uint64_t kept = ~0ull;
  if constexpr (GM != kNoGroups) {
    bool certain;
    if constexpr (GM == kGroupsInLds) {
      wave_fence();
      kept = pick_groups_lds<LANES, float>(val32, r, g, group_slack, certain);
      if (BY != kByLogit && !certain) {
        const double z = BY == kBySoftmax ? total64() : 1.0;
        wave_fence();
#pragma unroll
        for (int i = 0; i < EPL; ++i)
          if (held.has(i)) val[held.id(i)] = is_live(key[i]) ? choice64(x[i], b[i], z) : -__builtin_inf();
        wave_fence();
        kept = pick_groups_lds<LANES, double>(val, r, g, -1.f, certain);
      }
    } else {
      Two<float> two = two_of<EPL>(val_of);
      kept = pick_group_lanes<LANES>(two, r, g, group_slack, certain);
      if (BY != kByLogit && !certain) {
        // in f64, the experts that may be among their group's best: about one per lane
        const double z = BY == kBySoftmax ? total64() : 1.0;
        const float least = r.group_top > 1 && two.b != none ? two.b : two.a;
        const float limit = least - (group_slack + 0x1p-22f * fabsf(least));
        unsigned may = 0;
#pragma unroll
        for (int i = 0; i < EPL; ++i) may |= val_of[i] != none && val_of[i] >= limit ? 1u << i : 0u;
        Two<double> best{-__builtin_inf(), -__builtin_inf()};
        for (; may; may &= may - 1) {
          const int e = held.id(__ffs(may) - 1);
          best.add(choice64(l[e], bias ? bias[e] : 0.f, z));
        }
        kept = pick_group_lanes<LANES>(best, r, g, -1.f, certain);
      }
    }
    if constexpr (GM == kGroupsInLds) {
#pragma unroll
      for (int i = 0; i < EPL; ++i)
        // (& 63: ids past E may lie past group 63; they come behind every expert, kept or not)
        if (!((kept >> (((held.id(i) * r.inv_per) >> 20) & 63)) & 1)) key[i] = never_key();
    }
  }
  constexpr int L = EPL > 8 ? 8 : EPL;
  double list[L];
  best_keys<EPL, L>(key, list);
  // a lane whose head is never taken never moves up
  if (GM == kGroupLanes && !((kept >> (g >> (LANES == 32 ? r.share32 : r.share16))) & 1)) list[0] = never_key();
  const double end = L < EPL ? unknown_key() : never_key();
  my_e = 0;
  bool close = false, lost = false;  // choices too close to each other; more of them than were kept at hand
  float last = 0.f;
  for (int j = 0; j < r.k; ++j) {
    const double w = take_best<LANES, L>(list, end);
    lost |= w == unknown_key();
    if (BY != kByLogit && bias) {
      close |= j > 0 && !apart(last, key_value(w), slack);
      last = key_value(w);
    }
    if (g == j) my_e = key_id(w);
  }
  if (BY != kByLogit && bias) {
    // the candidates go on to the first one that is clearly behind
    int n = r.k;
    for (;; ++n) {
      const double w = take_best<LANES, L>(list, end);
      lost |= w == unknown_key();
      if (lost || apart(last, key_value(w), slack)) break;
      close = true;
      if (n == LANES) {
        lost = true;
        break;
      }
      last = key_value(w);
      if (g == n) my_e = key_id(w);
    }
    if (close && !lost) {
      // lane j's candidate, in f64, takes the slot of its rank
      const double z = BY == kBySoftmax ? total64() : 1.0;
      const double none64 = -__builtin_inf();
      double c = none64;
      int id = INT_MAX;
      if (g < n) {
        id = my_e;
        const float v = l[id], bv = bias[id];
        if (v - v == 0.f && bv - bv == 0.f) c = choice64(v, bv, z);
      }
      int rank = 0;
      others<LANES>(c, id, [&](double oc, int oid) { rank += oid != INT_MAX && (oc > c || (oc == c && oid < id)); });
      // lanes without a candidate keep to their own places behind
      rank = g < n ? rank : g;
      const int at = ((threadIdx.x & 63 & ~(LANES - 1)) + rank) * 4;
      my_e = __builtin_amdgcn_ds_permute(at, my_e);
    }
  }
  if (lost) my_e = select_exact<EPL, LANES, GM>(l, bias, r, g, val);

  // weights, from the chosen ones' scores in f64
  double s = 0.0;
  if (g < r.k) {
    const float v = l[my_e];
    const bool live = __builtin_isfinite(v) && (!bias || __builtin_isfinite(bias[my_e]));
    if (live) s = softmax ? exp((double)v - (double)top) : sigmoid64((double)v);
  }
  if (r.renorm) {
    const double sum = reduce<LANES>(s, [](double a, double b) { return a + b; });
    s = sum > 0.0 ? s / sum : 0.0;
  } else if (softmax) {
    s = sum_exp > 0.0 ? s / sum_exp : 0.0;  // 0: every expert masked
  }
  my_w = (float)(s * (double)r.scale);
}

// Tokens without queues.
template <int EPL, int LANES, int BY, int GM>
__global__ __launch_bounds__(64) void route_scored_kernel(const float* __restrict__ logits, int64_t ld,
                                                          const float* __restrict__ bias, int T, RouterArgs r,
                                                          int32_t* __restrict__ idx, float* __restrict__ w,
                                                          int32_t* __restrict__ flag) {
  extern __shared__ double vals[];
  const int g = threadIdx.x & (LANES - 1), tb = threadIdx.x / LANES;
  const int64_t t = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (64 / LANES) + tb;
  int e;
  float v;
  bool bad;
  // (the last tokens' lanes repeat the last one: a wave has no idle rows)
  route_scored<EPL, LANES, BY, GM>(logits, ld, bias, r, t < T ? t : T - 1, g, vals + tb * r.row, e, v, bad);
  if (t < T && g < r.k) {
    idx[t * r.k + g] = e;
    w[t * r.k + g] = v;
  }
  if (bad && flag) atomicOr(flag, kErrNonFinite);
}

// A fragment for the queues, 32 tokens per workgroup: routed, and each (token,
// slot) ranked among the workgroup's rows of its expert (as in k_route.hip: the
// tokens that picked an expert are a mask).  A fragment of one workgroup gets
// its queue entries and depths written here; else blockcnt [E][workgroups] gets
// the workgroup's rows per expert.
template <int EPL, int LANES, int BY, int GM>
__global__ __launch_bounds__(32 * LANES) void route_queue_kernel(
    const float* __restrict__ logits, const float* __restrict__ bias, int T, RouterArgs r, int32_t* __restrict__ r_idx,
    float* __restrict__ r_w, int32_t* __restrict__ r_rank, int32_t* __restrict__ blockcnt,
    int32_t* __restrict__ idx_out, float* __restrict__ w_out, AppendArgs a) {
  extern __shared__ double vals[];
  __shared__ uint32_t tok_mask[kMaxScoredExperts];
  const int tid = threadIdx.x, g = tid & (LANES - 1), tb = tid / LANES;
  const int t = blockIdx.x * 32 + tb;
  for (int e = tid; e < r.E; e += 32 * LANES) tok_mask[e] = 0;
  __syncthreads();
  int e;
  float w;
  bool bad;
  route_scored<EPL, LANES, BY, GM>(logits, r.E, bias, r, t < T ? t : T - 1, g, vals + tb * r.row, e, w, bad);
  const bool on = t < T && g < r.k;
  if (on) atomicOr(&tok_mask[e], 1u << tb);
  __syncthreads();
  const int rank = on ? __popc(tok_mask[e] & ((1u << tb) - 1u)) : 0;
  const int64_t o = (int64_t)t * r.k + g;
  if (on) {
    if (idx_out) idx_out[o] = e;
    if (w_out) w_out[o] = w;
  }
  if (bad) atomicOr(a.err, kErrNonFinite);
  if (gridDim.x == 1) {
    if (t < T) {
      const char* row = a.x + (int64_t)t * a.row_bytes;
      const int tok = token_id(t, g, r.k, a.token_base, a.token_ids, a.n_ids, a.live, a.pend, a.err);
      if (on) {
        QEntry en;
        en.row = row;
        en.token_slot = tok | (g << kTokenBits);
        en.w = w;
        a.q[(int64_t)e * a.q_stride + a.depth_cur[e] + rank] = en;
      }
      if (g == 0) a.tok_row[tok] = row;
    }
    for (int x = tid; x < r.E; x += 32 * LANES) a.depth_nxt[x] = a.depth_cur[x] + __popc(tok_mask[x]);
  } else {
    for (int x = tid; x < r.E; x += 32 * LANES) blockcnt[(int64_t)x * gridDim.x + blockIdx.x] = __popc(tok_mask[x]);
    if (on) {
      r_idx[o] = e;
      r_w[o] = w;
      r_rank[o] = rank;
    }
  }
}

// One wave per expert: its workgroup counts become the workgroups' first queue
// slots, and its depth after the fragment is published.
__global__ __launch_bounds__(64) void scan_scored_kernel(int32_t* __restrict__ blockcnt, int nb,
                                                         const int32_t* __restrict__ depth_cur,
                                                         int32_t* __restrict__ depth_nxt) {
  const int e = blockIdx.x, lane = threadIdx.x;
  int32_t* c = blockcnt + (int64_t)e * nb;
  int base = depth_cur[e];
  for (int b0 = 0; b0 < nb; b0 += 64) {
    const int b = b0 + lane;
    const int v = b < nb ? c[b] : 0;
    int x = v;  // inclusive scan
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(x, d);
      if (lane >= d) x += y;
    }
    if (b < nb) c[b] = base + x - v;
    base += __shfl(x, 63);
  }
  if (lane == 0) depth_nxt[e] = base;
}

// Queue entries of routed and ranked tokens, 32 per workgroup.  first: the
// scanned counts, or (direct) the counts themselves, of which every workgroup
// adds the ones before its own, and the last one publishes the depths.
__global__ __launch_bounds__(kRouteThreads) void append_scored_kernel(const int32_t* __restrict__ r_idx,
                                                                      const float* __restrict__ r_w,
                                                                      const int32_t* __restrict__ r_rank,
                                                                      const int32_t* __restrict__ first, bool direct,
                                                                      int T, int E, int k, AppendArgs a) {
  __shared__ int32_t base[kMaxScoredExperts];
  const int tid = threadIdx.x, nb = gridDim.x;
  for (int e = tid; e < E; e += kRouteThreads) {
    const int32_t* c = first + (int64_t)e * nb;
    int v = c[blockIdx.x];
    if (direct) {
      int sum = a.depth_cur[e];
#pragma unroll 8
      for (int b = 0; b < (int)blockIdx.x; ++b) sum += c[b];
      if ((int)blockIdx.x == nb - 1) a.depth_nxt[e] = sum + v;
      v = sum;
    }
    base[e] = v;
  }
  __syncthreads();
  const int g = tid & (kRouteLanes - 1);
  const int t = blockIdx.x * kRouteTokens + tid / kRouteLanes;
  if (t >= T) return;
  const char* row = a.x + (int64_t)t * a.row_bytes;
  const int tok = token_id(t, g, k, a.token_base, a.token_ids, a.n_ids, a.live, a.pend, a.err);
  if (g < k) {
    const int64_t o = (int64_t)t * k + g;
    const int e = r_idx[o];
    QEntry en;
    en.row = row;
    en.token_slot = tok | (g << kTokenBits);
    en.w = r_w[o];
    a.q[(int64_t)e * a.q_stride + base[e] + r_rank[o]] = en;
  }
  if (g == 0) a.tok_row[tok] = row;
}

// Calls f(EPL, LANES, BY, GM) as constants.
template <typename F>
static void by_rule(const RouterArgs& r, bool bias, F f) {
  using std::integral_constant;
  auto sized = [&](auto by, auto gm) {
    if (r.E <= 64)
      f(integral_constant<int, 4>{}, integral_constant<int, 16>{}, by, gm);
    else if (r.E <= 128)
      f(integral_constant<int, 8>{}, integral_constant<int, 16>{}, by, gm);
    else if (r.E <= 256)
      f(integral_constant<int, 16>{}, integral_constant<int, 16>{}, by, gm);
    else
      f(integral_constant<int, 16>{}, integral_constant<int, 32>{}, by, gm);
  };
  auto grouped = [&](auto by) {
    const int lanes = r.E <= 256 ? 16 : 32;
    if (r.n_groups == 1)
      sized(by, integral_constant<int, kNoGroups>{});
    else if (lanes % r.n_groups == 0 && r.E % lanes == 0)
      sized(by, integral_constant<int, kGroupLanes>{});
    else
      sized(by, integral_constant<int, kGroupsInLds>{});
  };
  if (!bias && !(r.n_groups > 1 && r.group_top > 1))
    grouped(integral_constant<int, kByLogit>{});
  else if (r.sigmoid)
    grouped(integral_constant<int, kBySigmoid>{});
  else
    grouped(integral_constant<int, kBySoftmax>{});
}

// Runs of experts per lane start and end at 16 bytes, in every row.
static int runs_aligned(const float* logits, int64_t ld, const float* bias, const RouterArgs& r) {
  const int lanes = r.E <= 256 ? 16 : 32;
  return (((uintptr_t)logits | (uintptr_t)bias) & 15) == 0 && ld % 4 == 0 && r.E % (4 * lanes) == 0;
}

hipError_t launch_route_scored(const float* logits, int64_t ld, const float* bias, int T, const RouterArgs& rule,
                               int32_t* idx, float* w, int32_t* flag, hipStream_t s) {
  RouterArgs r = rule;
  r.vec4 = runs_aligned(logits, ld, bias, r);
  by_rule(r, bias != nullptr, [&](auto epl, auto lanes, auto by, auto gm) {
    // a wave per workgroup: tokens spread over the CUs (256 threads: 64 tokens
    // 9.2 us instead of 7.4, 8192 and more within 1%)
    const int tokens = 64 / lanes();
    const size_t lds = gm() == kGroupsInLds ? (size_t)tokens * r.row * 8 : 0;
    const int64_t nb = (T + (int64_t)tokens - 1) / tokens, gx = nb < 1 << 24 ? nb : 1 << 24;
    // (a grid's side has fewer than 2^32 threads)
    route_scored_kernel<epl(), lanes(), by(), gm()>
        <<<dim3((unsigned)gx, (unsigned)((nb + gx - 1) / gx)), 64, lds, s>>>(logits, ld, bias, T, r, idx, w, flag);
  });
  return hipGetLastError();
}

hipError_t launch_route_queue(const float* logits, const float* bias, int T, const RouterArgs& rule, int32_t* r_idx,
                              float* r_w, int32_t* r_rank, int32_t* blockcnt, int32_t* idx_out, float* w_out,
                              const AppendArgs& a, hipStream_t s) {
  RouterArgs r = rule;
  r.vec4 = runs_aligned(logits, r.E, bias, r);
  const int nb = (T + 31) / 32;
  by_rule(r, bias != nullptr, [&](auto epl, auto lanes, auto by, auto gm) {
    const size_t lds = gm() == kGroupsInLds ? (size_t)32 * r.row * 8 : 0;
    route_queue_kernel<epl(), lanes(), by(), gm()><<<nb, 32 * lanes(), lds, s>>>(logits, bias, T, r, r_idx, r_w, r_rank, blockcnt,
                                                                         idx_out, w_out, a);
  });
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || nb == 1) return e;
  const bool direct = nb <= kDirectPrefixBlocks;
  if (!direct) {
    scan_scored_kernel<<<r.E, 64, 0, s>>>(blockcnt, nb, a.depth_cur, a.depth_nxt);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  append_scored_kernel<<<nb, kRouteThreads, 0, s>>>(r_idx, r_w, r_rank, blockcnt, direct, T, r.E, r.k, a);
  return hipGetLastError();
}

}  // namespace aep
