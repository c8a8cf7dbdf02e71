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

// Rows are shared out in one of two ways.
//
// Runs, for few rows: every row is cut into runs of nearly equal length, one workgroup each, none
// longer than `rounds` tiles for each of its waves: the smallest such number with which the runs
// of the batch fit the grid.  A workgroup then has one row only (to change rows in the middle
// costs it the latencies of a new start, which few others cover).
//
// smallest_rounds: count(q) is the number of runs of at most q tiles, for all rows; `tiles` those
// of all rows, `longest` of one; rows <= grid.
constexpr int kRoundsMin = 2;         // (a join of parts takes longer than one round more)
template <class Count>
AATC_PAGED_HD inline int smallest_rounds(int tiles, int longest, int rows, int grid, int waves,
                                         Count count) {
  int lo = (tiles + grid * waves - 1) / (grid * waves);          // the average: none lower fits
  if (lo < kRoundsMin) lo = kRoundsMin;
  if (count(lo * waves) <= grid) return lo;
  // A run for each row fits; and sum ceil(n / q) <= tiles / q + rows.
  int hi = (longest + waves - 1) / waves;
  if (grid > rows) {
    const int room = (grid - rows) * waves, closed = (tiles + room - 1) / room;
    hi = closed < hi ? closed : hi;
  }
  while (hi - lo > 1 + lo / 16) {                                // lo does not fit, hi does
    const int mid = (lo + hi) / 2;
    if (count(mid * waves) <= grid) hi = mid;
    else lo = mid;
  }
  return hi;
}
AATC_PAGED_HD inline int runs_of(int n, int q) { return (n + q - 1) / q; }
// Run i of `runs` has the row's tiles from here on.
AATC_PAGED_HD inline int run_begin(int n, int runs, int i) { return (int)((int64_t)n * i / runs); }

// Lines, for many rows: the tiles of all rows lie in one line, row after row; worker w (a wave for
// itself, or a workgroup whose waves share rows) takes those from w quota on, of several rows or
// of a part of one.  Or whole rows: a worker has one row (quota is then the longest).
//
// To begin a row, and to join its parts, takes a wave about as long as five tiles each.  So rows
// stay whole, a wave each, where there are waves enough and the longest is not much over the
// average share (1544 rows of 13 tiles at most: 57.4 us, 58.9 shared by workgroups), or a workgroup
// each.  Else waves for themselves, unless rows would be cut into many parts (784 rows of 60 tiles at
// most: 104.8 us by waves, 97.0 by workgroups).
struct LineWay {
  int quota;
  bool waves, whole;
};
AATC_PAGED_HD inline LineWay line_way(int tiles, int longest, int rows, int groups, int waves) {
  const int all = groups * waves, share = (tiles + all - 1) / all;
  if (rows <= all && longest <= share + 8) return {longest, true, true};
  if (rows <= groups && longest <= 8 * waves) return {longest, false, true};
  const int q = share > 4 ? share : 4;
  if (longest <= 3 * q) return {q, true, false};
  const int even = (tiles + groups - 1) / groups;
  return {even > waves ? even : waves, false, false};
}
// A row that starts at `start` with n tiles is shared by the workers first .. last.
struct RowShare {
  int first, last;
};
AATC_PAGED_HD inline RowShare row_share(int start, int n, int quota) {
  return {start / quota, (start + n - 1) / quota};
}
// The workspace slot of worker w's part of that row: one for a row that it goes on with, one
// for a row that it begins.
AATC_PAGED_HD inline int part_slot(int w, int start, int quota) {
  return 2 * w + (start >= w * quota ? 1 : 0);
}

}  // namespace aatc
