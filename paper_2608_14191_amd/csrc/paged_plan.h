// Which tokens of a sequence the paged attention reads, in tiles, and how the tiles of a batch
// are dealt to workgroups.  Plain C++, in every workgroup and on the host.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#define AATC_PAGED_HD __host__ __device__
#else
#define AATC_PAGED_HD
#endif

namespace aatc {

// Tiles of `tt` tokens that hold the attended tokens t < len, t >= len - window or t < sink
// (window 0: all): `head` tiles from token 0 on, then those from tile `skip` + head on.
struct RowTiles {
  int n, head, skip;
  AATC_PAGED_HD int token(int i, int tt) const { return (i < head ? i : i + skip) * tt; }
};

// At least one tile, also of an empty sequence: its workgroup writes the row's empty result.
AATC_PAGED_HD inline RowTiles row_tiles(int len, int window, int sink, int tt) {
  const int all = (len + tt - 1) / tt;
  const int lo = window > 0 && len > window ? len - window : 0;
  const int s = sink < lo ? sink : lo;
  const int head = (s + tt - 1) / tt, from = lo / tt;
  RowTiles r{all, head, 0};
  if (head < from) {
    r.skip = from - head;
    r.n = all - r.skip;
  }
  if (r.n < 1) r.n = 1;
  return r;
}

// Rows so short that one workgroup has each in a few rounds of its waves are not shared, if there
// is a workgroup for every row.
constexpr int kWholeRow = 32;
AATC_PAGED_HD inline bool rows_whole(int longest, int rows, int grid) {
  return longest <= kWholeRow && rows <= grid;
}

// Else: tiles of a workgroup, one for each of its waves at least.
constexpr int kQuotaMin = 8;
AATC_PAGED_HD inline int quota_of(int total, int grid) {
  const int even = (total + grid - 1) / grid;
  return even > kQuotaMin ? even : kQuotaMin;
}

// The tiles of all rows lie in one line, row after row; workgroup w takes those from w quota on.
// A row that starts at `start` with n tiles is shared by the workgroups first .. last.
struct RowShare {
  int first, last;
};
AATC_PAGED_HD inline RowShare row_share(int start, int n, int quota) {
  return {start / quota, (start + n - 1) / quota};
}
// The workspace slot of workgroup w's part of that row: one for a row that it goes on with, one
// for a row that it begins.
AATC_PAGED_HD inline int part_slot(int w, int start, int quota) {
  return 2 * w + (start >= w * quota ? 1 : 0);
}

}  // namespace aatc
