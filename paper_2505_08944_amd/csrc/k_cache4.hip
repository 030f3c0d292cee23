// Rows of keys and values into the pages of a cache in 4 bits, and back (cache4.h).
// Bound by HBM where there are many rows, else by the latency of the loads: the
// sequence's place, the page, the row.  Where sequences differ in their rows, a row's one is found by a scan of the
// ends before it, 64 per load: one row of each of 64 sequences 4.1 us, of 1024 9.5, of 4096 28.
#include <algorithm>
#include <climits>

#include "cache4.h"

namespace aep {

// The sequences of the 16 rows from t0 on, for the lanes of row r: those that end at or
// before a row are counted, 64 of them at a time.
__device__ __forceinline__ int seq_of_row(const Cache4Seqs& q, int t0, int r, int lane) {
  if (!q.rows) return (t0 + r) / q.n;
  int b = 0;
  for (int base = 0; base < q.batch; base += 64) {
    const int e = base + lane < q.batch ? q.rows[base + lane + 1] : INT_MAX;
    int n = 0, most = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int ends = __popcll(__ballot(e <= t0 + i));
      n = r == i ? ends : n;
      most = max(most, ends);
    }
    b += n;
    if (most < 64) break;
  }
  return b;
}

// One wave: 16 rows by four blocks of 32 values (of the heads' keys, then of their values), a quad of lanes
// for each row, eight values of each block in a lane.  So a quad reads, or writes, 64 consecutive bytes
// of a row, and 16 tokens in order fill a block's 256 bytes of keys, and lines of its values, in one
// store.  8168 rows of 8 heads of 128: written in 13.1 us, read in 10.7; with a wave per row 17.0 and 19.9.
template <int D, bool READ>
__global__ __launch_bounds__(256) void cache4_rows_kernel(const Cache4 c, const Cache4Seqs q, uint16_t* __restrict__ k,
                                                          uint16_t* __restrict__ v, int64_t k_row, int64_t k_head,
                                                          int64_t v_row, int64_t v_head) {
  constexpr int NB = D / 32, PIECE = D / 32;  // blocks; bytes of a token's values per lane
  const int lane = threadIdx.x & 63, r = lane >> 2, w = lane & 3;
  const uint32_t fours = (uint32_t)c.heads * NB / 2;  // groups of four blocks
  const uint64_t i = ((uint64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint64_t group = i >> 32 ? i / fours : (uint32_t)i / fours;
  if (group * 16 >= (uint64_t)q.total) return;
  const int t0 = (int)(group * 16), t = t0 + r, e0 = (int)(i - group * fours) * 4;
  if (i == 0 && q.rows && q.flag)  // (rows that descend may leave a row to nobody: all of them are looked at once)
    for (int j = lane; j < q.batch; j += 64)
      if (q.rows[j] < 0 || q.rows[j + 1] < q.rows[j] || q.rows[j + 1] > q.total) *q.flag = 1;
  // this lane's values of the blocks; those that are written are on their way while their place is looked up
  bool values[4];
  uint16_t* x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int e = e0 + j, hb = e >= c.heads * NB ? e - c.heads * NB : e, h = hb / NB, blk = hb % NB;
    const int row = min(t, q.total - 1);
    values[j] = e >= c.heads * NB;
    x[j] = (values[j] ? v + row * v_row + h * v_head : k + row * k_row + h * k_head) + blk * 32 + w * 8;
  }
  uint32_t raw[4][4];
  if constexpr (!READ)
#pragma unroll
    for (int j = 0; j < 4; ++j) __builtin_memcpy(raw[j], x[j], 16);
  const int b = seq_of_row(q, t0, r, lane);
  if (t >= q.total || b >= q.batch) return;  // behind the last sequence
  const SeqRows s = seq_rows(q, c.log_page, b);
  if (t < s.row0 || t - s.row0 >= s.n) return;
  int pos = s.len - s.n + t - s.row0;
  if constexpr (!READ) {
    // What has no place is left out: held to bounds, it would take another token's.  (No token of the sequence; rows
    // that are not all there; a token behind the last page.)
    pos += s.more;
    if (pos < 0 || !s.given || pos >> c.log_page >= q.max_pages) return;
  }
  int page = 0;
  if (pos >= 0) {
    const int p = q.pages[b * q.ld_pages + (pos >> c.log_page)];
    page = page_in(q, c.n_pages, p);
    if (!READ && p != page) return;
  }
  const int at = pos & ((1 << c.log_page) - 1);
  const int place = cache4_place(at & 31);

  // of each block, where this lane's codes are, and the scale
  uint8_t *codes[4], *scale[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int e = e0 + j, hb = values[j] ? e - c.heads * NB : e, blk = hb % NB;
    const int64_t head = (int64_t)page * c.heads + hb / NB;
    const int part = D == 256 ? (w >> 1) * 256 + (w & 1) * 4 : w * 128;
    codes[j] = values[j] ? c.v + (((head << c.log_page) + (at & ~31)) * D >> 1) + (blk * (512 / D) * 32 + place) * PIECE + part
                         : c.k + (((head << c.log_page) + (at & ~15)) * D >> 1) + blk * 256 + (at & 15) * 16 + w * 4;
    scale[j] = values[j] ? c.vs + ((head << c.log_page) + (at & ~31)) * NB + blk * 32 + place
                         : c.ks + ((head << c.log_page) + at) * NB + blk;
  }
  if constexpr (READ) {
    uint32_t in[4] = {0, 0, 0, 0}, sb[4] = {127, 127, 127, 127};
    if (pos >= 0) {  // (zeros where the sequence has no token)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (D == 64 && values[j])
          in[j] = (uint32_t)*reinterpret_cast<const uint16_t*>(codes[j]) |
                  (uint32_t)*reinterpret_cast<const uint16_t*>(codes[j] + 64) << 16;
        else
          in[j] = *reinterpret_cast<const uint32_t*>(codes[j]);
        sb[j] = *scale[j];
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<uint4*>(x[j]) = mx4_bf16x8(in[j], mx4_scale(sb[j]));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float u[8];
      uint32_t big = 0;
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        u[2 * n] = bf16_lo(raw[j][n]);
        u[2 * n + 1] = bf16_hi(raw[j][n]);
        big = max(big, max(raw[j][n] << 16 & 0x7fffffffu, raw[j][n] & 0x7fff0000u));
      }
      big = quad_max(big);
      const uint32_t sb = mx4_scale_byte(big);
      const uint32_t out = mx4_codes(u, mx4_scale(sb == kMx4NaN ? 127 : sb));
      if (D == 64 && values[j]) {
        *reinterpret_cast<uint16_t*>(codes[j]) = (uint16_t)out;
        *reinterpret_cast<uint16_t*>(codes[j] + 64) = (uint16_t)(out >> 16);
      } else {
        *reinterpret_cast<uint32_t*>(codes[j]) = out;
      }
      if (w == 0) *scale[j] = (uint8_t)sb;
    }
  }
}

template <bool READ>
static hipError_t rows_launch(const Cache4& c, const Cache4Seqs& q, uint16_t* k, uint16_t* v, int64_t k_row, int64_t k_head,
                              int64_t v_row, int64_t v_head, hipStream_t s) {
  const int64_t waves = ((int64_t)q.total + 15) / 16 * ((int64_t)c.heads * (c.d / 32) / 2), blocks = (waves + 3) / 4;
  const int64_t gx = std::min<int64_t>(blocks, 1 << 22);
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
