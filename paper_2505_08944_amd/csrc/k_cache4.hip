// Rows of keys and values into the pages of a cache in 4 bits, and back (cache4.h).
// Bound by HBM where there are many rows, else by the latency of the loads: the
// sequence's place, the page, the row.
#include <algorithm>
#include <climits>

#include "cache4.h"

namespace aep {

// The sequence of row t, found by all lanes of a wave: the sequences that end at or
// before it are counted, 64 of them at a time.
__device__ __forceinline__ int seq_of_row(const Cache4Seqs& q, int t, int lane) {
  if (!q.rows) return t / q.n;
  int b = 0;
  for (int base = 0; base < q.batch; base += 64) {
    const int e = base + lane < q.batch ? q.rows[base + lane + 1] : INT_MAX;
    const int n = __popcll(__ballot(e <= t));
    b += n;
    if (n < 64) break;
  }
  return b;
}

// One wave per row: its lanes have a block of 32 each of the heads of keys, then of values.
template <int D, bool READ>
__global__ __launch_bounds__(256) void cache4_rows_kernel(const Cache4 c, const Cache4Seqs q, uint16_t* __restrict__ k,
                                                          uint16_t* __restrict__ v, int64_t k_row, int64_t k_head,
                                                          int64_t v_row, int64_t v_head) {
  constexpr int NB = D / 32, PIECE = D / 32;  // blocks; bytes of a token's values per lane
  const int lane = threadIdx.x & 63;
  const int t = __builtin_amdgcn_readfirstlane((int)((blockIdx.y * gridDim.x + blockIdx.x) * 4 + (threadIdx.x >> 6)));
  if (t >= q.total || t < 0) return;
  if (t == 0 && q.rows && q.flag)  // (rows that descend may leave a row to nobody: all of them are looked at once)
    for (int i = lane; i < q.batch; i += 64)
      if (q.rows[i] < 0 || q.rows[i + 1] < q.rows[i] || q.rows[i + 1] > q.total) *q.flag = 1;
  const int b = seq_of_row(q, t, lane);
  if (b >= q.batch) return;  // behind the last sequence
  const SeqRows s = seq_rows(q, c.log_page, b);
  const int i = t - s.row0, pos = s.len - s.n + i;
  if (i < 0 || i >= s.n) return;
  const int items = 2 * c.heads * NB;
  if (pos < 0) {  // no token of the sequence
    if constexpr (READ)
      for (int e = lane; e < items; e += 64) {
        const bool values = e >= c.heads * NB;
        const int hb = values ? e - c.heads * NB : e, h = hb / NB, blk = hb % NB;
        uint4* o = reinterpret_cast<uint4*>((values ? v + t * v_row + h * v_head : k + t * k_row + h * k_head) + blk * 32);
#pragma unroll
        for (int w = 0; w < 4; ++w) o[w] = make_uint4(0, 0, 0, 0);
      }
    return;
  }
  const int page = seq_page(q, c.n_pages, b, pos >> c.log_page), at = pos & ((1 << c.log_page) - 1);
  const int place = cache4_place(at & 31);
  for (int e = lane; e < items; e += 64) {
    const bool values = e >= c.heads * NB;
    const int hb = values ? e - c.heads * NB : e, h = hb / NB, blk = hb % NB;
    const int64_t head = (int64_t)page * c.heads + h;
    uint16_t* x = (values ? v + t * v_row + h * v_head : k + t * k_row + h * k_head) + blk * 32;
    // codes of the block: 16 bytes of a key, or 32 / (D / 16) pieces of values, 32 places apart
    uint8_t* codes = values ? c.v + (((head << c.log_page) + (at & ~31)) * D >> 1) + (blk * (512 / D) * 32 + place) * PIECE
                            : c.k + (((head << c.log_page) + (at & ~15)) * D >> 1) + blk * 256 + (at & 15) * 16;
    uint8_t* scale = values ? c.vs + ((head << c.log_page) + (at & ~31)) * NB + blk * 32 + place
                            : c.ks + ((head << c.log_page) + at) * NB + blk;
    uint32_t w[4];
    if constexpr (READ) {
      if (!values) {
        *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(codes);
      } else if constexpr (D == 64) {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(codes);
#pragma unroll
        for (int m = 0; m < 4; ++m) w[m] = (uint32_t)p[m * 64] | (uint32_t)p[m * 64 + 32] << 16;
      } else {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(codes);
#pragma unroll
        for (int m = 0; m < 4; ++m) w[m] = D == 128 ? p[m * 32] : p[(m >> 1) * 64 + (m & 1)];
      }
      const float f = mx4_scale(*scale);
#pragma unroll
      for (int m = 0; m < 4; ++m) reinterpret_cast<uint4*>(x)[m] = mx4_bf16x8(w[m], f);
    } else {
      uint32_t in[16];
      __builtin_memcpy(in, x, 64);
      uint32_t big = 0;
#pragma unroll
      for (int m = 0; m < 16; ++m) big = max(big, max(in[m] << 16 & 0x7fffffffu, in[m] & 0x7fff0000u));
      const uint32_t sb = mx4_scale_byte(big);
      const float f = mx4_scale(sb == kMx4NaN ? 127 : sb);
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        float u[8];
#pragma unroll
        for (int n = 0; n < 8; ++n) u[n] = n & 1 ? bf16_hi(in[m * 4 + (n >> 1)]) : bf16_lo(in[m * 4 + (n >> 1)]);
        w[m] = mx4_codes(u, f);
      }
      *scale = (uint8_t)sb;
      if (!values) {
        *reinterpret_cast<uint4*>(codes) = make_uint4(w[0], w[1], w[2], w[3]);
      } else if constexpr (D == 64) {
        uint16_t* p = reinterpret_cast<uint16_t*>(codes);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          p[m * 64] = (uint16_t)w[m];
          p[m * 64 + 32] = (uint16_t)(w[m] >> 16);
        }
      } else {
        uint32_t* p = reinterpret_cast<uint32_t*>(codes);
#pragma unroll
        for (int m = 0; m < 4; ++m) p[D == 128 ? m * 32 : (m >> 1) * 64 + (m & 1)] = w[m];
      }
    }
  }
}

template <bool READ>
static hipError_t rows_launch(const Cache4& c, const Cache4Seqs& q, uint16_t* k, uint16_t* v, int64_t k_row, int64_t k_head,
                              int64_t v_row, int64_t v_head, hipStream_t s) {
  const int64_t blocks = ((int64_t)q.total + 3) / 4, gx = std::min<int64_t>(blocks, 1 << 22);
  const dim3 g((unsigned)gx, (unsigned)((blocks + gx - 1) / gx));
  if (c.d == 64) cache4_rows_kernel<64, READ><<<g, 256, 0, s>>>(c, q, k, v, k_row, k_head, v_row, v_head);
  if (c.d == 128) cache4_rows_kernel<128, READ><<<g, 256, 0, s>>>(c, q, k, v, k_row, k_head, v_row, v_head);
  if (c.d == 256) cache4_rows_kernel<256, READ><<<g, 256, 0, s>>>(c, q, k, v, k_row, k_head, v_row, v_head);
  return hipGetLastError();
}

hipError_t launch_cache4_append(const Cache4& c, const Cache4Seqs& q, const uint16_t* k, const uint16_t* v, int64_t k_row,
                                int64_t k_head, int64_t v_row, int64_t v_head, hipStream_t s) {
  return rows_launch<false>(c, q, const_cast<uint16_t*>(k), const_cast<uint16_t*>(v), k_row, k_head, v_row, v_head, s);
}

hipError_t launch_cache4_read(const Cache4& c, const Cache4Seqs& q, uint16_t* k, uint16_t* v, hipStream_t s) {
  const int64_t row = (int64_t)c.heads * c.d;
  return rows_launch<true>(c, q, k, v, row, c.d, row, c.d, s);
}

}  // namespace aep
