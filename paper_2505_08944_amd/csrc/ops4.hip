// Host side of the calls on 4-bit data: the quantiser, the dense product with 4-bit
// weights, the cache of keys and values and the attention over it.
#include <algorithm>
#include <climits>

#include "cache4.h"
#include "linear4.h"
#include "ops.h"

using namespace aep;

namespace {

hipStream_t stream_of(void* s) { return reinterpret_cast<hipStream_t>(s); }
aep_status launched(hipError_t e) { return e == hipSuccess ? AEP_OK : AEP_ERR_DEVICE; }
int value_size(int32_t t) { return t == AEP_F32 ? 4 : 2; }
aep_status check_dtype(int32_t t) {
  if (t < AEP_F32 || t > AEP_FP8_E4M3) return AEP_ERR_INVALID_ARG;
  return t == AEP_FP8_E4M3 ? AEP_ERR_UNSUPPORTED : AEP_OK;
}

aep_status check_matrix(int64_t rows, int32_t k, int64_t ld, int32_t dtype) {
  if (rows < 0 || k < 1 || ld < k) return AEP_ERR_INVALID_ARG;
  if (const aep_status st = check_dtype(dtype); st != AEP_OK) return st;
  if (k > 1 << 30 || rows > ((int64_t)1 << 38) / ((k + 31) / 32)) return AEP_ERR_UNSUPPORTED;
  return AEP_OK;
}

aep_status check_weights(int32_t n, int32_t k) {
  if (n < 1 || k < 1) return AEP_ERR_INVALID_ARG;
  return n > 1 << 30 || k > 1 << 30 || (int64_t)n * k > (int64_t)1 << 40 ? AEP_ERR_UNSUPPORTED : AEP_OK;
}

aep_status check_linear4(const aep_linear4_desc* l) {
  if (!l || l->m < 0) return AEP_ERR_INVALID_ARG;
  if (const aep_status st = check_weights(l->n, l->k); st != AEP_OK) return st;
  if (l->fn < AEP_FN_NONE || l->fn > AEP_FN_GELU_TANH) return AEP_ERR_INVALID_ARG;
  if (l->ldx < l->k || l->ldy < l->n) return AEP_ERR_INVALID_ARG;
  for (int32_t t : {l->y_dtype, l->bias_dtype, l->res_dtype})
    if (const aep_status st = check_dtype(t); st != AEP_OK) return st;
  if (l->m > 1 << 30 || (int64_t)l->m * l->n > (int64_t)1 << 38) return AEP_ERR_UNSUPPORTED;
  return AEP_OK;
}

LinearArgs linear4_args(const aep_linear4_desc& l, const void* x, const void* packed, const void* bias, const void* residual,
                        void* y) {
  aep_linear_desc d{};
  d.m = l.m;
  d.n = l.n;
  d.k = l.k;
  d.x_dtype = d.w_dtype = AEP_BF16;
  d.y_dtype = l.y_dtype;
  d.bias_dtype = l.bias_dtype;
  d.res_dtype = l.res_dtype;
  d.fn = l.fn;
  d.ldx = l.ldx;
  d.ldw = (l.k + 7) / 8 * 8;
  d.ldy = l.ldy;
  d.ldr = l.ldr;
  return linear_args(d, x, packed, nullptr, bias, residual, y);
}

bool linear4_misaligned(const aep_linear4_desc& l, const void* x, const void* residual, const void* y) {
  return off(x, 2) || off(residual, value_size(l.res_dtype)) || off(y, value_size(l.y_dtype));
}

// ------------------------------------------------------------------- cache
aep_status check_cache(const aep_cache4* c) {
  if (!c || c->n_pages < 1 || c->n_heads < 1 || c->page_size < 1 || c->head_dim < 1) return AEP_ERR_INVALID_ARG;
  if (c->page_size & (c->page_size - 1) || c->page_size < 32 || c->page_size > 4096) return AEP_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return AEP_ERR_UNSUPPORTED;
  if (c->n_heads > 1024 || (int64_t)c->n_pages * c->page_size * c->n_heads > (int64_t)1 << 38) return AEP_ERR_UNSUPPORTED;
  return AEP_OK;
}
int64_t cache_values(const aep_cache4& c) { return (int64_t)c.n_pages * c.page_size * c.n_heads * c.head_dim; }
Cache4 cache_of(const aep_cache4& c, void* mem) {
  const int64_t n = cache_values(c);
  Cache4 o{};
  o.k = reinterpret_cast<uint8_t*>(mem);
  o.v = o.k + n / 2;
  o.ks = o.v + n / 2;
  o.vs = o.ks + n / 32;
  o.n_pages = c.n_pages;
  o.log_page = __builtin_ctz(c.page_size);
  o.heads = c.n_heads;
  o.d = c.head_dim;
  return o;
}

aep_status check_seqs(const aep_cache4& c, const aep_cache4_seqs* s) {
  if (!s || s->batch < 0 || s->total < 0 || s->max_pages < 0 || s->ld_pages < s->max_pages) return AEP_ERR_INVALID_ARG;
  if (s->batch == 0 && s->total > 0 && !s->rows) return AEP_ERR_INVALID_ARG;
  if (!s->rows && s->batch && s->total % s->batch) return AEP_ERR_INVALID_ARG;
  if (s->total && s->batch && (!s->lens || (s->max_pages && !s->pages))) return AEP_ERR_INVALID_ARG;
  if (off(s->pages, 4) || off(s->lens, 4) || off(s->rows, 4) || off(s->flag, 4)) return AEP_ERR_INVALID_ARG;
  if (s->total > 1 << 30 || s->batch > 1 << 24 || (int64_t)s->max_pages * c.page_size > 1 << 30) return AEP_ERR_UNSUPPORTED;
  return AEP_OK;
}
Cache4Seqs seqs_of(const aep_cache4_seqs& s) {
  Cache4Seqs o{};
  o.pages = s.pages;
  o.lens = s.lens;
  o.rows = s.rows;
  o.ld_pages = s.ld_pages;
  o.max_pages = s.max_pages;
  o.batch = s.batch;
  o.total = s.total;
  o.n = s.batch ? s.total / s.batch : 0;
  o.flag = s.flag;
  return o;
}

// Rows of heads of d values that do not overlap, whichever of the two goes first.  (Counts below 2^31 and distances up to
// 2^40: their products are more than 64 bits hold.)
bool apart(int64_t rows, int64_t row, int64_t heads, int64_t head, int64_t d) {
  const auto fits = [&](int64_t n1, int64_t s1, int64_t n2, int64_t s2) {
    return (n1 < 2 || s1 >= d) && (n2 < 2 || s2 >= (n1 < 2 ? 0 : (__int128)(n1 - 1) * s1) + d);
  };
  return fits(heads, head, rows, row) || fits(rows, row, heads, head);
}

aep_status check_attend(const aep_cache4* c, const aep_cache4_seqs* s, const aep_attend4_desc* a) {
  if (const aep_status st = check_cache(c); st != AEP_OK) return st;
  if (const aep_status st = check_seqs(*c, s); st != AEP_OK) return st;
  if (!a || a->n_heads < 1 || a->n_heads % c->n_heads || a->window < 0 || a->max_rows < 0) return AEP_ERR_INVALID_ARG;
  if (!(a->scale > 0.f) || !(a->scale <= 0x1p127f)) return AEP_ERR_INVALID_ARG;  // (times log2 e it is finite)
  const int64_t most = (int64_t)1 << 40;
  if (a->q_row < 0 || a->q_head < 0 || a->out_row < 0 || a->out_head < 0) return AEP_ERR_INVALID_ARG;
  if (a->q_row > most || a->q_head > most || a->out_row > most || a->out_head > most) return AEP_ERR_UNSUPPORTED;
  if (!apart(s->total, a->out_row, a->n_heads, a->out_head, c->head_dim)) return AEP_ERR_INVALID_ARG;
  const int64_t cols = (int64_t)s->total * a->n_heads, len = (int64_t)s->max_pages * c->page_size;
  // (units of work are counted in 31 bits)
  if (cols > 1 << 30 ||
      (cols / 16 + (int64_t)(s->batch + 1) * c->n_heads) * (len / 128 + 2) >= (int64_t)1 << 31)
    return AEP_ERR_UNSUPPORTED;
  return AEP_OK;
}
Attend4Plan plan_of(const aep_cache4& c, const aep_cache4_seqs& s, const aep_attend4_desc& a) {
  return attend4_plan(s.batch, s.total, s.rows != nullptr, a.max_rows ? a.max_rows : s.total, c.n_heads, a.n_heads / c.n_heads,
                      c.head_dim, (int64_t)s.max_pages * c.page_size, persistent_workgroups());
}

}  // namespace

extern "C" {

aep_status aep_mx4_quantize(const void* x, int32_t x_dtype, int64_t ldx, int64_t rows, int32_t k, void* codes, void* scale,
                            void* stream) {
  if (const aep_status st = check_matrix(rows, k, ldx, x_dtype); st != AEP_OK) return st;
  if (rows == 0) return AEP_OK;
  if (!x || !codes || !scale || off(x, value_size(x_dtype))) return AEP_ERR_INVALID_ARG;
  return launched(launch_mx4_quantize(x, x_dtype, ldx, rows, k, reinterpret_cast<uint8_t*>(codes),
                                      reinterpret_cast<uint8_t*>(scale), stream_of(stream)));
}

aep_status aep_mx4_dequantize(const void* codes, const void* scale, int64_t rows, int32_t k, void* y, int32_t y_dtype,
                              int64_t ldy, void* stream) {
  if (const aep_status st = check_matrix(rows, k, ldy, y_dtype); st != AEP_OK) return st;
  if (rows == 0) return AEP_OK;
  if (!y || !codes || !scale || off(y, value_size(y_dtype))) return AEP_ERR_INVALID_ARG;
  return launched(launch_mx4_dequantize(reinterpret_cast<const uint8_t*>(codes), reinterpret_cast<const uint8_t*>(scale), rows,
                                        k, y, y_dtype, ldy, stream_of(stream)));
}

aep_status aep_linear4_packed_bytes(int32_t n, int32_t k, size_t* bytes) {
  if (const aep_status st = check_weights(n, k); st != AEP_OK) return st;
  if (!bytes) return AEP_ERR_INVALID_ARG;
  *bytes = (size_t)linear4_pieces(n, k) * kLinear4Piece;
  return AEP_OK;
}

aep_status aep_linear4_pack(const void* codes, const void* scale, int32_t n, int32_t k, void* packed, void* stream) {
  if (const aep_status st = check_weights(n, k); st != AEP_OK) return st;
  if (!codes || !scale || !packed || off(packed, 16)) return AEP_ERR_INVALID_ARG;
  return launched(launch_linear4_pack(reinterpret_cast<const uint8_t*>(codes), reinterpret_cast<const uint8_t*>(scale), n, k,
                                      reinterpret_cast<uint8_t*>(packed), stream_of(stream)));
}

aep_status aep_linear4_workspace(const aep_linear4_desc* l, const void* x, const void* residual, const void* y, size_t* bytes) {
  if (const aep_status st = check_linear4(l); st != AEP_OK) return st;
  if (!bytes || linear4_misaligned(*l, x, residual, y)) return AEP_ERR_INVALID_ARG;
  *bytes = 0;
  if (l->m == 0) return AEP_OK;
  const LinearArgs p = linear4_args(*l, x, nullptr, nullptr, residual, const_cast<void*>(y));
  const Linear4Plan r = linear4_plan(p, persistent_workgroups(), INT64_MAX);
  if (r.widen) *bytes = (size_t)r.bytes();
  return AEP_OK;
}

aep_status aep_linear4(const aep_linear4_desc* l, const void* x, const void* packed, const void* bias, const void* residual,
                       void* y, void* d_ws, size_t ws_bytes, void* stream) {
  if (const aep_status st = check_linear4(l); st != AEP_OK) return st;
  if (residual && l->ldr < l->n) return AEP_ERR_INVALID_ARG;
  if (l->m == 0) return AEP_OK;
  if (!x || !packed || !y) return AEP_ERR_INVALID_ARG;
  if (linear4_misaligned(*l, x, residual, y) || off(packed, 16) || off(bias, value_size(l->bias_dtype)) || off(d_ws, 16))
    return AEP_ERR_INVALID_ARG;
  // y may be the residual, element for element, and nothing else of it
  if (residual == y && (l->res_dtype != l->y_dtype || (l->ldr != l->ldy && l->m > 1))) return AEP_ERR_INVALID_ARG;
  const LinearArgs p = linear4_args(*l, x, packed, bias, residual, y);
  return launched(launch_linear4(p, persistent_workgroups(), d_ws, (int64_t)std::min<size_t>(ws_bytes, INT64_MAX / 2),
                                 stream_of(stream)));
}

aep_status aep_cache4_bytes(const aep_cache4* c, size_t* bytes) {
  if (const aep_status st = check_cache(c); st != AEP_OK) return st;
  if (!bytes) return AEP_ERR_INVALID_ARG;
  const int64_t n = cache_values(*c);
  *bytes = (size_t)(n + n / 16);
  return AEP_OK;
}

aep_status aep_cache4_append(const aep_cache4* c, void* mem, const aep_cache4_seqs* s, const void* k, int64_t k_row,
                             int64_t k_head, const void* v, int64_t v_row, int64_t v_head, void* stream) {
  if (const aep_status st = check_cache(c); st != AEP_OK) return st;
  if (const aep_status st = check_seqs(*c, s); st != AEP_OK) return st;
  if (k_row < 0 || k_head < 0 || v_row < 0 || v_head < 0) return AEP_ERR_INVALID_ARG;
  if (std::max({k_row, k_head, v_row, v_head}) > (int64_t)1 << 40) return AEP_ERR_UNSUPPORTED;
  if (s->total == 0 || s->batch == 0) return AEP_OK;
  if (!mem || off(mem, 16) || !k || !v || off(k, 2) || off(v, 2)) return AEP_ERR_INVALID_ARG;
  return launched(launch_cache4_append(cache_of(*c, mem), seqs_of(*s), reinterpret_cast<const uint16_t*>(k),
                                       reinterpret_cast<const uint16_t*>(v), k_row, k_head, v_row, v_head, stream_of(stream)));
}

aep_status aep_cache4_read(const aep_cache4* c, const void* mem, const aep_cache4_seqs* s, void* k, void* v, void* stream) {
  if (const aep_status st = check_cache(c); st != AEP_OK) return st;
  if (const aep_status st = check_seqs(*c, s); st != AEP_OK) return st;
  if (s->total == 0 || s->batch == 0) return AEP_OK;
  if (!mem || off(mem, 16) || !k || !v || off(k, 16) || off(v, 16)) return AEP_ERR_INVALID_ARG;
  return launched(launch_cache4_read(cache_of(*c, const_cast<void*>(mem)), seqs_of(*s), reinterpret_cast<uint16_t*>(k),
                                     reinterpret_cast<uint16_t*>(v), stream_of(stream)));
}

aep_status aep_cache4_attend_workspace(const aep_cache4* c, const aep_cache4_seqs* s, const aep_attend4_desc* a, size_t* bytes) {
  if (const aep_status st = check_attend(c, s, a); st != AEP_OK) return st;
  if (!bytes) return AEP_ERR_INVALID_ARG;
  *bytes = s->total && s->batch ? (size_t)plan_of(*c, *s, *a).bytes : 0;
  return AEP_OK;
}

aep_status aep_cache4_attend(const aep_cache4* c, const void* mem, const aep_cache4_seqs* s, const aep_attend4_desc* a,
                             const void* q, void* out, float* lse, void* d_ws, size_t ws_bytes, void* stream) {
  if (const aep_status st = check_attend(c, s, a); st != AEP_OK) return st;
  if (s->total == 0 || s->batch == 0) return AEP_OK;
  if (!mem || off(mem, 16) || !q || !out || off(q, 2) || off(out, 2) || off(lse, 4) || off(d_ws, 16)) return AEP_ERR_INVALID_ARG;
  const Attend4Plan p = plan_of(*c, *s, *a);
  if (!d_ws || ws_bytes < (size_t)p.bytes) return AEP_ERR_CAPACITY;
  Attend4Args g{};
  g.c = cache_of(*c, const_cast<void*>(mem));
  g.s = seqs_of(*s);
  g.q = reinterpret_cast<const uint16_t*>(q);
  g.out = reinterpret_cast<uint16_t*>(out);
  g.lse = lse;
  g.q_row = a->q_row;
  g.q_head = a->q_head;
  g.o_row = a->out_row;
  g.o_head = a->out_head;
  g.group = a->n_heads / c->n_heads;
  g.window = a->window >= (int64_t)s->max_pages * c->page_size ? 0 : a->window;
  g.scale = (float)((double)a->scale * 1.4426950408889634);
  g.parts = reinterpret_cast<float*>(d_ws);
  for (int i = 0; i < p.passes; ++i) {
    g.nc = p.pass[i].nc;
    g.workers = p.pass[i].workers;
    g.over = p.pass[i].over;
    g.most = p.pass[i].most;
    g.units = p.pass[i].units;
    if (launch_attend4(g, stream_of(stream)) != hipSuccess) return AEP_ERR_DEVICE;
  }
  return AEP_OK;
}

}  // extern "C"
