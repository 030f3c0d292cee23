// The tile kernel's device code on the host (linear_host.py), thread by thread,
// with ffn_host.cpp's recorder in place of the hardware.
#include "recorder.inc"

#define __host__
static const void* kernarg;
#define __builtin_amdgcn_kernarg_segment_ptr() (kernarg)
#define __builtin_amdgcn_exp2f(x) exp2f(x)
struct TwoWords {
  unsigned operator[](int) const { return 0; }
};
#define __builtin_amdgcn_raw_buffer_load_b64(...) (TwoWords{})

#include "linear_device.inc"

using namespace aep;

// As for the FFN: two accesses of the same bytes, one or both of them loads, must
// be apart, with a barrier between them where they are of different waves.
static bool ordered(const Access& r, const Access& w) {
  if (r.wave == w.wave) return r.done_seq < w.issue_seq || w.done_seq < r.issue_seq;
  return r.done < w.issue || w.done < r.issue;
}

// The chain of items that workgroup (xcd, 0) of 8 runs of a product of K = k
// values: `whole` rounds of 256 x 256 tiles, then `rest` tiles cut into halves and
// p0 pieces, then `lrow` rows of tiles of family fam in pr pieces.  Returns the
// unordered pairs, the first of them in msg; -1 where waves pass different numbers
// of barriers.
template <bool FP8>
static long violations(int k, int whole, int rest, int halves, int p0, int fam, int lrow, int pr, int xcd, long* n_reads,
                       char* msg, int msg_n) {
  static std::vector<unsigned char> mem(kTileLds);
  lds_mem = mem.data();
  reads.assign(kTileLds / 16, {});
  writes.assign(kTileLds / 16, {});
  const int nwg = 8;
  TileParams t{};
  LinearCut& c = t.cut;
  c.ncol = 4;
  c.whole = whole * nwg;
  c.rest = rest;
  c.nrow = (c.whole + c.rest + 3) / 4;
  c.halves = halves;
  c.p0 = p0;
  c.fam = fam;
  c.lrow = lrow;
  c.pr = pr;
  LinearArgs& p = t.a;
  p.n = 1024;
  p.m = c.nrow * 256 + lrow * (256 >> fam);
  p.k = k;
  p.ldx = p.ldw = (k + 15) / 16 * 16;
  p.ldy = p.n;
  p.wide = kWideBf16;
  static uint16_t scale[2048];
  p.scale = FP8 ? scale : nullptr;
  p.w_dtype = FP8 ? kFP8 : kBF16;
  c.items = c.whole + c.rest_items() + c.last_tiles(p.n) * c.pr;
  std::vector<float> scratch(c.floats(p.n) + 1);
  t.scratch = scratch.data();
  kernarg = &t;

  int barriers = -1;
  bool uneven = false;
  for (int tid = 0; tid < 512; ++tid) {
    threadIdx.x = (unsigned)tid;
    epoch = seq = 0;
    vm.clear();
    rd_pend.clear();
    fl_pend.clear();
    int r = 0;
    int item = linear_nth(the_cut(), r, nwg, xcd, 0);
    while (item >= 0) {
      const int kind = linear_kind(the_cut(), item);
      if (kind == 0)
        run_shape<FP8, 0, 2>(lds_mem, 0, nwg, xcd, 0, r, item);
      else if (kind == 1)
        run_shape<FP8, 0, 1>(lds_mem, 0, nwg, xcd, 0, r, item);
      else if (kind == 2)
        run_shape<FP8, 1, 1>(lds_mem, 0, nwg, xcd, 0, r, item);
      else
        run_shape<FP8, 2, 1>(lds_mem, 0, nwg, xcd, 0, r, item);
    }
    if (barriers >= 0 && epoch != barriers) uneven = true;
    barriers = epoch;
  }
  if (uneven) return -1;
  long bad = 0;
  *n_reads = 0;
  for (size_t a = 0; a < reads.size(); ++a) {
    *n_reads += (long)reads[a].size();
    for (const Access& x : reads[a])
      for (const Access& w : writes[a])
        if (!ordered(x, w) && bad++ == 0)
          snprintf(msg, msg_n, "LDS byte %zu: read by wave %d in slot %d .. %d, loaded by wave %d in slot %d .. %d", a * 16,
                   x.wave, x.issue, x.done, w.wave, w.issue, w.done);
    for (const Access& x : writes[a])
      for (const Access& w : writes[a])
        if (x.wave < w.wave && !ordered(x, w) && bad++ == 0)
          snprintf(msg, msg_n, "LDS byte %zu: loaded by wave %d in slot %d .. %d and by wave %d in slot %d .. %d", a * 16,
                   x.wave, x.issue, x.done, w.wave, w.issue, w.done);
  }
  return bad;
}

extern "C" long linear_order_violations(int fp8, int k, const int* c, int xcd, long* n_reads, char* msg, int msg_n) {
  return fp8 ? violations<true>(k, c[0], c[1], c[2], c[3], c[4], c[5], c[6], xcd, n_reads, msg, msg_n)
             : violations<false>(k, c[0], c[1], c[2], c[3], c[4], c[5], c[6], xcd, n_reads, msg, msg_n);
}
