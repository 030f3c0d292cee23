// The paged cache of keys and values in 4 bits (mx4.h): its layout, and what its
// kernels share.
//
// A page holds P tokens (a power of two, 32 at least) of every head.  D values of a
// head are D / 32 blocks.  In the order in which the attention's lanes take them:
//   keys     [page][head][P / 16][block][16 tokens][16 bytes]: the codes in their order
//   values   [page][head][P / 32][16 l][4 g][8 j][D / 32 bytes]: the D / 16 codes from
//            D / 16 l on of token cache4_token(g, j) of the 32
//   scales of keys    [page][head][P][block]
//   scales of values  [page][head][P / 32][block][4 g][8 j]
// one behind the other.  No byte belongs to two tokens.
#pragma once

#include "aep_internal.h"
#include "attend4_plan.h"
#include "mx4.h"

namespace aep {

struct Cache4 {
  uint8_t *k, *v, *ks, *vs;
  int n_pages, log_page, heads, d;
};

// Where sequences' rows and tokens are: row i of the n rows of sequence b is its
// token len - n + i, which lies in page pages[b][token / P].  Sequence b has the rows
// from rows[b] to rows[b + 1]; without rows, n rows each.
struct Cache4Seqs {
  const int32_t *pages, *lens, *rows;
  int64_t ld_pages;
  int max_pages, batch, total, n;
  int32_t* flag;
};

// What the device reads is held to what the buffers have; what had to be is reported.
struct SeqRows {
  int row0, n, len;
  int more;    // tokens behind the last page, which len is without
  bool given;  // the rows are as they were given
};
__device__ __forceinline__ SeqRows seq_rows(const Cache4Seqs& q, int log_page, int b) {
  SeqRows s;
  s.given = true;
  if (q.rows) {
    const int a = q.rows[b], e = q.rows[b + 1];
    s.row0 = min(max(a, 0), q.total);
    const int last = min(max(e, s.row0), q.total);
    s.n = last - s.row0;
    s.given = a == s.row0 && e == last;
    if (q.flag && !s.given) *q.flag = 1;
  } else {
    s.row0 = b * q.n;
    s.n = q.n;
  }
  const int l = q.lens[b];
  s.len = (int)min((int64_t)max(l, 0), (int64_t)q.max_pages << log_page);
  s.more = max(l, 0) - s.len;
  if (q.flag && l != s.len && s.n) *q.flag = 1;  // (without rows, nothing needs it)
  return s;
}
__device__ __forceinline__ int page_in(const Cache4Seqs& q, int n_pages, int p) {
  const int in = min(max(p, 0), n_pages - 1);
  if (q.flag && p != in) *q.flag = 1;
  return in;
}
// The same entry of a wave, not held to bounds yet: through the scalar cache, so that whoever waits
// for it does not wait for the vector loads in flight.
__device__ __forceinline__ int seq_page_raw(const Cache4Seqs& q, int b, int i) {
  typedef const __attribute__((address_space(4))) int32_t* table;
  return reinterpret_cast<table>(reinterpret_cast<uintptr_t>(q.pages))[b * q.ld_pages + i];
}

// Place (g, j) of token t of 32: the rows 4 g + i of an MFMA's result over tokens 0 ..
// 15 are a lane's values j = i, those over 16 .. 31 its values j = 4 + i.
__device__ __forceinline__ int cache4_place(int t) { return ((t & 15) >> 2) * 8 + (t & 3) + (t >> 4) * 4; }

struct Attend4Args {
  Cache4 c;
  Cache4Seqs s;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  int64_t q_row, q_head, o_row, o_head;
  int group;    // heads of queries per head of the cache
  int window;
  int over, most;  // sequences of more than `over` columns (a row and a head of a group each), at most `most`
  float scale;     // times log2 e
  int workers, nc, units;  // (units: at most, of rows that ascend)
  // Scratch: two parts of a tile for each workgroup (of the tile that its share begins inside
  // of, and of the one that begins in its share and goes on behind it), 16 nc columns of D sums, a
  // reference and a sum of weights each; then what the second launch has to know of the latter.
  float* parts;
  struct Shared {
    int last;  // its last workgroup (0: there is no such tile)
    int total, head, tile, cols, row0, pos0, pad;
  };
  __host__ __device__ Shared* shared() const {
    return reinterpret_cast<Shared*>(parts + (int64_t)workers * 2 * (16 * nc) * (c.d + 2));
  }
};
hipError_t launch_attend4(const Attend4Args& a, hipStream_t s);
hipError_t launch_cache4_append(const Cache4& c, const Cache4Seqs& q, const uint16_t* k, const uint16_t* v, int64_t k_row,
                                int64_t k_head, int64_t v_row, int64_t v_head, hipStream_t s);
hipError_t launch_cache4_read(const Cache4& c, const Cache4Seqs& q, uint16_t* k, uint16_t* v, hipStream_t s);

}  // namespace aep
