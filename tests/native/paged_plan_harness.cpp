// Plain C entry points to csrc/paged_plan.h for the CPU tests.
#include "paged_plan.h"

using namespace aatc;

extern "C" {

// Tokens of the row's tiles into out (room for `room`); returns their number.
int tiles(int len, int window, int sink, int tt, int* out, int room) {
  const RowTiles r = row_tiles(len, window, sink, tt);
  for (int i = 0; i < r.n && i < room; ++i) out[i] = r.token(i, tt);
  return r.n;
}

int rounds(const int* n, int batch, int rows, int grid, int waves) {
  int tiles = 0, longest = 0;
  for (int b = 0; b < batch; ++b) {
    tiles += n[b] * rows;
    longest = n[b] > longest ? n[b] : longest;
  }
  return smallest_rounds(tiles, longest, batch * rows, grid, waves, [&](int q) {
    int c = 0;
    for (int b = 0; b < batch; ++b) c += rows * runs_of(n[b], q);
    return c;
  });
}

int run_at(int n, int runs, int i) { return run_begin(n, runs, i); }

void way(int tiles, int longest, int rows, int groups, int waves, int* out) {
  const LineWay w = line_way(tiles, longest, rows, groups, waves);
  out[0] = w.quota;
  out[1] = w.waves;
  out[2] = w.whole;
}

void share(int start, int n, int quota, int* out) {
  const RowShare s = row_share(start, n, quota);
  out[0] = s.first;
  out[1] = s.last;
}

int slot(int w, int start, int quota) { return part_slot(w, start, quota); }
}
