// Routing by scores: softmax or sigmoid scores, a bias for the choice, expert
// groups, top-k, weights from the scores of the chosen (the rule is stated at
// aep_router in aep.h).
//
// Choices are compared in binary64: a sigmoid plus a bias of like size has
// neighbours that binary32 cannot tell apart, and the same logits must give
// the same experts on every rank.
#include <float.h>
#include <limits.h>

#include "aep_internal.h"
#include "route_token_id.h"

namespace aep {

// The larger key, equal: the lower id; id INT_MAX: none.
__device__ __forceinline__ void better(double& v, int& e, double ov, int oe) {
  if (oe != INT_MAX && (e == INT_MAX || ov > v || (ov == v && oe < e))) {
    v = ov;
    e = oe;
  }
}
__device__ __forceinline__ void wave_best(double& v, int& e) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) better(v, e, __shfl_xor(v, d), __shfl_xor(e, d));
}

// One wave per token; lane l holds experts l, l + 64, ...
template <int EPL>
__global__ __launch_bounds__(256) void route_scored_kernel(const float* __restrict__ logits, int64_t ld,
                                                           const float* __restrict__ bias, int T, RouterArgs r,
                                                           int32_t* __restrict__ idx, float* __restrict__ w,
                                                           int32_t* __restrict__ idx2, float* __restrict__ w2,
                                                           int32_t* __restrict__ flag) {
  __shared__ double worth[4][EPL * 64];  // an expert's value to its group
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t t = (int64_t)blockIdx.x * 4 + wave;
  const bool valid = t < T;
  const int E = r.E, per = E / r.n_groups;
  double key[EPL], score[EPL];
  bool live[EPL];
  bool bad = false;
  float l[EPL];
  float top = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int e = i * 64 + lane;
    l[i] = valid && e < E ? logits[t * ld + e] : -__builtin_inff();
    live[i] = __builtin_isfinite(l[i]);
    if (!live[i] && l[i] != -__builtin_inff()) bad = true;
    if (live[i]) top = fmaxf(top, l[i]);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  double total = 0.0;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    score[i] = 0.0;
    if (live[i]) score[i] = r.sigmoid ? 1.0 / (1.0 + exp(-(double)l[i])) : exp((double)l[i] - (double)top);
    total += score[i];
  }
  if (!r.sigmoid) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d);
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (live[i]) score[i] = score[i] / total;
  }
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int e = i * 64 + lane;
    double c = bias ? score[i] + (e < E ? (double)bias[e] : 0.0) : (double)l[i];
    if (live[i] && !__builtin_isfinite(c)) {
      live[i] = false;
      score[i] = 0.0;
      bad = true;
    }
    key[i] = live[i] ? c : -__builtin_inf();
    worth[wave][e] = !live[i] ? -__builtin_inf() : bias || r.group_top > 1 ? score[i] + (bias ? (double)bias[e] : 0.0) : (double)l[i];
  }
  __syncthreads();

  // groups: lane g holds group g's value
  uint64_t kept = ~0ull;
  if (r.n_groups > 1) {
    double v = -__builtin_inf();
    if (lane < r.n_groups) {
      double second = -__builtin_inf();
      for (int i = 0; i < per; ++i) {
        const double x = worth[wave][lane * per + i];
        if (x > v) {
          second = v;
          v = x;
        } else if (x > second) {
          second = x;
        }
      }
      if (r.group_top > 1 && second != -__builtin_inf()) v += second;
    }
    kept = 0;
    for (int j = 0; j < r.top_groups; ++j) {
      double bv = v;
      int be = lane < r.n_groups && !((kept >> lane) & 1) ? lane : INT_MAX;
      wave_best(bv, be);
      kept |= 1ull << be;
    }
  }
  unsigned avail = 0;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int e = i * 64 + lane;
    if (e < E && (r.n_groups == 1 || ((kept >> (e / per)) & 1))) avail |= 1u << i;
  }
  double my_s = 0.0, sum = 0.0;
  int my_e = 0;
  for (int j = 0; j < r.k; ++j) {
    double bv = -__builtin_inf(), bs = 0.0;
    int be = INT_MAX;
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if ((avail >> i) & 1) better(bv, be, key[i], i * 64 + lane);
    wave_best(bv, be);
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (be == i * 64 + lane) {
        bs = score[i];
        avail &= ~(1u << i);
      }
    bs = __shfl(bs, be & 63);
    sum += bs;
    if (lane == j) {
      my_e = be;
      my_s = bs;
    }
  }
  if (r.renorm) my_s = sum > 0.0 ? my_s / sum : 0.0;
  if (valid && lane < r.k) {
    const int64_t o = t * r.k + lane;
    const float v = (float)(my_s * (double)r.scale);
    idx[o] = my_e;
    w[o] = v;
    if (idx2) idx2[o] = my_e;
    if (w2) w2[o] = v;
  }
  if (bad && flag) atomicOr(flag, kErrNonFinite);
}

// Rank of each (token, slot) among its block's rows of the same expert, and
// the block's rows per expert: blockcnt [E][nb].
__global__ __launch_bounds__(kRouteThreads) void rank_scored_kernel(const int32_t* __restrict__ r_idx, int T, int E,
                                                                    int k, int32_t* __restrict__ r_rank,
                                                                    int32_t* __restrict__ blockcnt) {
  __shared__ uint32_t tok_mask[kMaxScoredExperts];
  const int tid = threadIdx.x, g = tid & (kRouteLanes - 1), tb = tid / kRouteLanes;
  const int t = blockIdx.x * kRouteTokens + tb;
  const bool on = t < T && g < k;
  for (int e = tid; e < E; e += kRouteThreads) tok_mask[e] = 0;
  __syncthreads();
  const int64_t o = (int64_t)t * k + g;
  const int e = on ? r_idx[o] : 0;
  if (on) atomicOr(&tok_mask[e], 1u << tb);
  __syncthreads();
  for (int x = tid; x < E; x += kRouteThreads) blockcnt[(int64_t)x * gridDim.x + blockIdx.x] = __popc(tok_mask[x]);
  if (on) r_rank[o] = __popc(tok_mask[e] & ((1u << tb) - 1u));
}

// One wave per expert: its block counts become the blocks' first queue slots,
// and its depth after the fragment is published.
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

__global__ __launch_bounds__(kRouteThreads) void append_scored_kernel(
    const int32_t* __restrict__ r_idx, const float* __restrict__ r_w, const int32_t* __restrict__ r_rank,
    const int32_t* __restrict__ first, int T, int k, const char* x, int64_t row_bytes, int32_t token_base,
    QEntry* __restrict__ q, int64_t q_stride, const void** __restrict__ tok_row, const int32_t* __restrict__ token_ids,
    int n_ids, int32_t* __restrict__ live, int32_t* __restrict__ pend, int32_t* __restrict__ err) {
  const int tid = threadIdx.x, g = tid & (kRouteLanes - 1);
  const int t = blockIdx.x * kRouteTokens + tid / kRouteLanes;
  if (t >= T) return;
  const char* row = x + (int64_t)t * row_bytes;
  const int tok = token_id(t, g, k, token_base, token_ids, n_ids, live, pend, err);
  if (g < k) {
    const int64_t o = (int64_t)t * k + g;
    const int e = r_idx[o];
    QEntry en;
    en.row = row;
    en.token_slot = tok | (g << kTokenBits);
    en.w = r_w[o];
    q[(int64_t)e * q_stride + first[(int64_t)e * gridDim.x + blockIdx.x] + r_rank[o]] = en;
  }
  if (g == 0) tok_row[tok] = row;
}

hipError_t launch_route_scored(const float* logits, int64_t ld, const float* bias, int T, const RouterArgs& r,
                               int32_t* idx, float* w, int32_t* idx2, float* w2, int32_t* flag, hipStream_t s) {
  const int nb = (int)(((int64_t)T + 3) / 4);
  if (r.E <= 64)
    route_scored_kernel<1><<<nb, 256, 0, s>>>(logits, ld, bias, T, r, idx, w, idx2, w2, flag);
  else if (r.E <= 128)
    route_scored_kernel<2><<<nb, 256, 0, s>>>(logits, ld, bias, T, r, idx, w, idx2, w2, flag);
  else if (r.E <= 256)
    route_scored_kernel<4><<<nb, 256, 0, s>>>(logits, ld, bias, T, r, idx, w, idx2, w2, flag);
  else
    route_scored_kernel<8><<<nb, 256, 0, s>>>(logits, ld, bias, T, r, idx, w, idx2, w2, flag);
  return hipGetLastError();
}

hipError_t launch_append_scored(const int32_t* r_idx, const float* r_w, int32_t* r_rank, int32_t* blockcnt, int T, int E,
                                int k, const char* x, int64_t row_bytes, int32_t token_base, const int32_t* depth_cur,
                                int32_t* depth_nxt, QEntry* q, int64_t q_stride, const void** tok_row,
                                const int32_t* token_ids, int n_ids, int32_t* live, int32_t* pend, int32_t* err,
                                hipStream_t s) {
  const int nb = (T + kRouteTokens - 1) / kRouteTokens;
  rank_scored_kernel<<<nb, kRouteThreads, 0, s>>>(r_idx, T, E, k, r_rank, blockcnt);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  scan_scored_kernel<<<E, 64, 0, s>>>(blockcnt, nb, depth_cur, depth_nxt);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  append_scored_kernel<<<nb, kRouteThreads, 0, s>>>(r_idx, r_w, r_rank, blockcnt, T, k, x, row_bytes, token_base, q,
                                                    q_stride, tok_row, token_ids, n_ids, live, pend, err);
  return hipGetLastError();
}

}  // namespace aep
