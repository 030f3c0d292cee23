// Host side of the calls that need no context: the dense product and routing
// without queues.
#include <algorithm>
#include <atomic>
#include <climits>
#include <cmath>

#include "linear_tiles.h"
#include "ops.h"

using namespace aep;

namespace aep {

aep_status check_router(const aep_router* r) {
  if (!r) return AEP_ERR_INVALID_ARG;
  if (r->n_experts < 1 || r->top_k < 1 || r->top_k > r->n_experts) return AEP_ERR_INVALID_ARG;
  if (r->score != AEP_SCORE_SOFTMAX && r->score != AEP_SCORE_SIGMOID) return AEP_ERR_INVALID_ARG;
  if (r->n_groups < 1 || r->n_groups > kMaxRouteGroups || r->n_experts % r->n_groups) return AEP_ERR_INVALID_ARG;
  if (r->top_groups < 1 || r->top_groups > r->n_groups) return AEP_ERR_INVALID_ARG;
  if ((int64_t)r->top_groups * (r->n_experts / r->n_groups) < r->top_k) return AEP_ERR_INVALID_ARG;
  if (r->group_top != 1 && r->group_top != 2) return AEP_ERR_INVALID_ARG;
  if (r->renorm != 0 && r->renorm != 1) return AEP_ERR_INVALID_ARG;
  if (!std::isfinite(r->scale) || !(r->scale > 0.f)) return AEP_ERR_INVALID_ARG;
  if (r->n_experts > kMaxScoredExperts || r->top_k > kMaxScoredTopK) return AEP_ERR_UNSUPPORTED;
  return AEP_OK;
}

RouterArgs router_args(const aep_router& r) {
  RouterArgs a{};
  a.E = r.n_experts;
  a.k = r.top_k;
  a.sigmoid = r.score == AEP_SCORE_SIGMOID;
  a.n_groups = r.n_groups;
  a.top_groups = r.top_groups;
  a.group_top = r.group_top;
  a.renorm = r.renorm;
  a.scale = r.scale;
  a.per = r.n_experts / r.n_groups;
  a.inv_per = ((1 << 20) + a.per - 1) / a.per;
  while ((r.n_groups << (a.share16 + 1)) <= 16) ++a.share16;
  while ((r.n_groups << (a.share32 + 1)) <= 32) ++a.share32;
  a.row = r.n_experts | 1;  // (odd: tokens start in different banks)
  return a;
}

static int esize(int32_t t) { return t == AEP_F32 ? 4 : t == AEP_BF16 ? 2 : 1; }

LinearArgs linear_args(const aep_linear_desc& l, const void* x, const void* w, const void* scale, const void* bias,
                       const void* residual, void* y) {
  const int xs = esize(l.x_dtype), ws = esize(l.w_dtype);
  LinearArgs p{};
  p.m = l.m;
  p.n = l.n;
  p.k = l.k;
  p.x_dtype = l.x_dtype;
  p.w_dtype = l.w_dtype;
  p.y_dtype = l.y_dtype;
  p.bias_dtype = l.bias_dtype;
  p.res_dtype = l.res_dtype;
  p.fn = l.fn;
  p.ldx = l.ldx;
  p.ldw = l.ldw;
  p.ldy = l.ldy;
  p.ldr = l.ldr;
  p.x = x;
  p.w = w;
  p.scale = scale;
  p.bias = bias;
  p.res = residual;
  p.y = y;
  p.x_aligned = !off(x, 16) && (l.ldx * xs) % 16 == 0;
  p.w_aligned = !off(w, 16) && (l.ldw * ws) % 16 == 0;
  p.aligned = p.x_aligned && p.w_aligned && ((int64_t)l.k * xs) % 16 == 0 && ((int64_t)l.k * ws) % 16 == 0;
  const bool f32_res = l.res_dtype == AEP_F32;
  if (l.y_dtype == AEP_BF16 && l.n % 8 == 0 && !off(y, 16) && l.ldy % 8 == 0 &&
      (!residual || (!f32_res && !off(residual, 16) && l.ldr % 8 == 0)))
    p.wide = kWideBf16;
  // (a tile's offsets fit 31 bits)
  if (l.y_dtype == AEP_F32 && l.n % 4 == 0 && l.ldy < 1 << 21 &&
      (!residual || (f32_res ? l.ldr < 1 << 21 : !off(residual, 4) && l.ldr % 2 == 0)))
    p.wide = kWideF32;
  return p;
}

// One workgroup per CU of the current device, a multiple of the 8 XCDs.
int persistent_workgroups() {
  constexpr int kDevices = 64;
  static std::atomic<int> seen[kDevices];  // 0: not asked yet
  int dev = -1, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kDevices) return 256;
  if ((n = seen[dev].load(std::memory_order_relaxed)) > 0) return n;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return 256;
  n = ffn_grid(n);
  seen[dev].store(n, std::memory_order_relaxed);
  return n;
}

}  // namespace aep

namespace {


aep_status check_linear(const aep_linear_desc* l) {
  if (!l || l->m < 0 || l->n < 1 || l->k < 1) return AEP_ERR_INVALID_ARG;
  const int32_t types[] = {l->x_dtype, l->w_dtype, l->y_dtype, l->bias_dtype, l->res_dtype};
  for (int32_t t : types)
    if (t < AEP_F32 || t > AEP_FP8_E4M3) return AEP_ERR_INVALID_ARG;
  if (l->fn < AEP_FN_NONE || l->fn > AEP_FN_GELU_TANH) return AEP_ERR_INVALID_ARG;
  if (l->ldx < l->k || l->ldw < l->k || l->ldy < l->n) return AEP_ERR_INVALID_ARG;
  const bool f32 = l->x_dtype == AEP_F32 && l->w_dtype == AEP_F32 && l->y_dtype == AEP_F32;
  const bool bf = l->x_dtype == AEP_BF16 && (l->w_dtype == AEP_BF16 || l->w_dtype == AEP_FP8_E4M3) &&
                  (l->y_dtype == AEP_BF16 || l->y_dtype == AEP_F32);
  if (!f32 && !bf) return AEP_ERR_UNSUPPORTED;
  if (l->bias_dtype == AEP_FP8_E4M3 || l->res_dtype == AEP_FP8_E4M3) return AEP_ERR_UNSUPPORTED;
  // indices and tile counts are 32-bit (an output of 2^38 values does not fit any GPU)
  if (std::max({l->m, l->n, l->k}) > 1 << 30 || (int64_t)l->m * l->n > (int64_t)1 << 38) return AEP_ERR_UNSUPPORTED;
  return AEP_OK;
}

// Bytes of scratch of the cut that is taken where there is enough.
size_t linear_scratch(const aep_linear_desc& l, const void* x, const void* w, const void* residual, const void* y) {
  if (l.m == 0) return 0;
  const LinearArgs p = linear_args(l, x, w, nullptr, nullptr, residual, const_cast<void*>(y));
  const TilesPlan t = linear_tiles_plan(p, persistent_workgroups(), INT64_MAX);
  return t.use ? (size_t)t.bytes(p.n) : 0;
}

}  // namespace

extern "C" {

aep_status aep_route_topk(const aep_router* r, const float* logits, int64_t ld_logits, const float* bias, int32_t T,
                          int32_t* idx, float* w, int32_t* flag, void* stream) {
  const aep_status st = check_router(r);
  if (st != AEP_OK) return st;
  if (T < 0 || ld_logits < r->n_experts) return AEP_ERR_INVALID_ARG;
  if (T == 0) return AEP_OK;
  if (!logits || !idx || !w) return AEP_ERR_INVALID_ARG;
  if (off(logits, 4) || off(bias, 4) || off(idx, 4) || off(w, 4) || off(flag, 4)) return AEP_ERR_INVALID_ARG;
  return launch_route_scored(logits, ld_logits, bias, T, router_args(*r), idx, w, flag,
                             reinterpret_cast<hipStream_t>(stream)) == hipSuccess
             ? AEP_OK
             : AEP_ERR_DEVICE;
}

aep_status aep_linear_workspace(const aep_linear_desc* l, size_t* bytes) {
  const aep_status st = check_linear(l);
  if (st != AEP_OK) return st;
  if (!bytes) return AEP_ERR_INVALID_ARG;
  const void* const some = reinterpret_cast<const void*>(16);
  *bytes = std::max(linear_scratch(*l, some, some, nullptr, some), linear_scratch(*l, some, some, some, some));
  return AEP_OK;
}

aep_status aep_linear_workspace_at(const aep_linear_desc* l, const void* x, const void* w, const void* residual,
                                   const void* y, size_t* bytes) {
  const aep_status st = check_linear(l);
  if (st != AEP_OK) return st;
  if (!bytes) return AEP_ERR_INVALID_ARG;
  if (off(x, esize(l->x_dtype)) || off(w, esize(l->w_dtype)) || off(residual, esize(l->res_dtype)) ||
      off(y, esize(l->y_dtype)))
    return AEP_ERR_INVALID_ARG;
  *bytes = linear_scratch(*l, x, w, residual, y);
  return AEP_OK;
}

aep_status aep_linear(const aep_linear_desc* l, const void* x, const void* w, const void* scale, const void* bias,
                      const void* residual, void* y, void* d_ws, size_t ws_bytes, void* stream) {
  const aep_status st = check_linear(l);
  if (st != AEP_OK) return st;
  if (residual && l->ldr < l->n) return AEP_ERR_INVALID_ARG;
  if (l->m == 0) return AEP_OK;
  if (!x || !w || !y) return AEP_ERR_INVALID_ARG;
  if ((l->w_dtype == AEP_FP8_E4M3) != (scale != nullptr)) return AEP_ERR_INVALID_ARG;
  if (off(x, esize(l->x_dtype)) || off(w, esize(l->w_dtype)) || off(y, esize(l->y_dtype)) || off(scale, 2) ||
      off(bias, esize(l->bias_dtype)) || off(residual, esize(l->res_dtype)) || off(d_ws, 16))
    return AEP_ERR_INVALID_ARG;
  // y may be the residual, element for element, and nothing else of it
  if (residual == y && (l->res_dtype != l->y_dtype || (l->ldr != l->ldy && l->m > 1))) return AEP_ERR_INVALID_ARG;
  const LinearArgs p = linear_args(*l, x, w, scale, bias, residual, y);
  return launch_linear(p, persistent_workgroups(), reinterpret_cast<float*>(d_ws),
                       d_ws ? (int64_t)std::min<size_t>(ws_bytes / 4, INT64_MAX / 4) : 0,
                       reinterpret_cast<hipStream_t>(stream)) == hipSuccess
             ? AEP_OK
             : AEP_ERR_DEVICE;
}

}  // extern "C"
