// Which kernels run the attention over a cache in 4 bits (k_attend4.hip), with how many workgroups (host).
#pragma once

#include <stdint.h>

#include <algorithm>
#include <climits>

namespace aep {

constexpr int kAttendUnit = 128;   // tokens
constexpr int kAttendWide = 8;     // columns in 16s of the kernel for many
constexpr int kAttendShared = 32;  // bytes of Attend4Args::Shared
// Workgroups per CU, which are waves per SIMD: as many as registers allow without spilling.
constexpr int attend_per_cu(int d, int nc) { return d * nc == 64 ? 4 : d * nc == 128 ? 3 : d * nc == 256 ? 2 : 1; }

// The attention's launches: each takes the sequences of more than `over` columns and at most `most`, with
// tiles of nc 16 columns and so many workgroups; bytes of scratch, which they use one after the other.
// units: as many as sequences of disjoint rows can have (fewer than 2^31 by the caller's checks).
struct Attend4Plan {
  int passes;
  struct {
    int nc, workers, over, most, units;
  } pass[2];
  int64_t bytes;
};

// rows: whether sequences differ in their rows, of which one has at most max_rows.
// Tiles of 16 columns for sequences of up to 16, else of 32; the kernel for many for those of more
// than 64, if its workgroups have 8 units each at least (its parts are four times as large).  us, the
// kernel for many and tiles of 32, 4 heads of 128 in the cache, 32 sequences of up to 8192 tokens: 32 columns
// 53 and 41, 64 61 and 65, 128 72 and 98, 256 113 and 169; 4 sequences: 64 35 and 28, 256 51 and 37.
// The lengths lie on the device: max_len is what the table of pages has room for, and of a table that is wider than its
// longest sequence the rule expects more units than there are.  us, a table of 8192 tokens (or 131072) and one as wide as
// the sequences, 8 heads of 128: 4 x 64 rows of 1000 tokens 52 and 29, 32 x 32 of 300 37 and 28, 4 x 100 of 300 28 and
// 26, 1 x 300 of 300 23 and 27, 8 x 600 of 600 77 and 77.
// Sequences that differ in their rows are taken by both kinds, one after the other, unless none can have
// many (64 of up to 8192 tokens, one with 512 rows, the others with one, 4 heads to one of the cache: 169;
// by the one kind 196, by the other 241).
inline Attend4Plan attend4_plan(int batch, int total, bool rows, int max_rows, int heads, int group, int d, int64_t max_len, int ncu) {
  constexpr int kFew = 64, kUnitsOfMany = 8;
  Attend4Plan p{};
  const int64_t each = rows ? std::min(max_rows, total) : total / std::max(batch, 1), most = each * group;  // columns
  const auto units = [&](int nc) {
    return heads * ((int64_t)total * group / (16 * nc) + batch) * std::max<int64_t>(1, (max_len + kAttendUnit - 1) / kAttendUnit);
  };
  const auto per_cu = [&](int nc) { return nc < kAttendWide ? attend_per_cu(d, nc) : d == 256 ? 1 : 2; };
  const auto add = [&](int nc, int over, int upto) {
    const int workers = (int)std::min<int64_t>((units(nc) + 7) / 8 * 8, (int64_t)ncu * per_cu(nc));
    p.pass[p.passes].nc = nc;
    p.pass[p.passes].workers = workers;
    p.pass[p.passes].over = over;
    p.pass[p.passes].most = upto;
    p.pass[p.passes].units = (int)units(nc);
    ++p.passes;
    p.bytes = std::max(p.bytes, (int64_t)workers * ((int64_t)2 * (16 * nc) * (d + 2) * 4 + kAttendShared));
  };
  const bool many = most > kFew && units(kAttendWide) >= (int64_t)ncu * per_cu(kAttendWide) * kUnitsOfMany;
  if (!many || rows) add(most <= 16 || (many && group <= 16) ? 1 : 2, 0, many ? kFew : INT_MAX);
  if (many) add(kAttendWide, rows ? kFew : 0, INT_MAX);
  return p;
}

}  // namespace aep
