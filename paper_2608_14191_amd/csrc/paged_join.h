// What the workgroups of a row of the attention over pages have of it, joined, and what a row ends as.
// Device code.
#pragma once

#include <hip/hip_runtime.h>

#include "paged.h"
#include "paged_tile.h"
#include "params.h"

namespace aatc {
namespace {

constexpr int kPagedHeads = 16;                   // query heads of a row

// What one wave has of a row: for head n of its lanes the maximum, the sum and the value sums
// (acc[j][r]: channel M::channel(j, r, g)) over the tiles first, first + step .. below last.
struct RowPart {
  float m, l;
  v4f acc[8];
};

// LDS of the joins: the waves' sums, then (the same bytes) the weights of a row's parts; and the
// sums over groups of them.
template <int W, int GROUPS>
struct JoinSpace {
  union {
    float sums[W][kPagedHeads][kD + 4];            // (rows padded: banks)
    struct {
      float m[kPagedHeads][GROUPS], l[kPagedHeads][GROUPS];
    } parts;
  };
  v4f groups[64 * W];
  float m[W][kPagedHeads], l[W][kPagedHeads];
  float top[kPagedHeads], total[kPagedHeads];
};

// Joins the parts of a row in their order (slot(p, h, offset): 16 bytes of part p of head h):
// weights first, a wave to a head, then the sums of (head, four channels) units by groups of
// threads, whose first loads are on their way meanwhile.
template <int W, int GROUPS, class Finish, class Slot>
__device__ inline void join_parts(JoinSpace<W, GROUPS>& sh, int parts, int heads, Finish finish,
                                  Slot slot) {
  constexpr int NT = 64 * W, U = 8;                // U loads in flight
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int units = heads * (kD / 4);
  v4f x[U];
  int width = min(units, NT), groups = NT / width;
  int unit = tid % width, grp = tid / width;
  auto issue = [&](int p0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int p = p0 + u * groups;
      x[u] = ((grp < groups) & (p < parts)) ? slot(p, unit / (kD / 4), 16 + 16 * (unit % (kD / 4)))
                                            : (v4f){0.f, 0.f, 0.f, 0.f};
    }
  };
  issue(grp);
  for (int i = tid; i < heads * parts; i += NT) {
    const int h = i % heads, p = i / heads;
    const v4f ml = slot(p, h, 0);
    sh.parts.m[h][p] = ml[0];
    sh.parts.l[h][p] = ml[1];
  }
  __syncthreads();
  for (int h = wave; h < heads; h += W) {
    float m = -INFINITY, l = 0.f;
    for (int p = lane; p < parts; p += 64)
      if (sh.parts.l[h][p] != 0.f) m = fmaxf(m, sh.parts.m[h][p]);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    const float ref = m == -INFINITY ? 0.f : m;
    for (int p = lane; p < parts; p += 64) {
      const float pl = sh.parts.l[h][p];
      const float w = pl == 0.f ? 0.f : __builtin_amdgcn_exp2f(sh.parts.m[h][p] - ref);
      l += pl == 0.f ? 0.f : w * pl;               // (NaN stays)
      sh.parts.m[h][p] = w;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) l += __shfl_xor(l, o, 64);
    if (lane == 0) {
      sh.top[h] = m;
      sh.total[h] = l;
    }
  }
  __syncthreads();
  for (int base = 0;;) {
    const int h = unit / (kD / 4);
    v4f acc = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = grp;;) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int p = p0 + u * groups;
        const float w = ((grp < groups) & (p < parts)) ? sh.parts.m[h][p] : 0.f;
        acc += w * x[u];
      }
      p0 += U * groups;
      if (p0 - grp >= parts) break;                // (uniform)
      issue(p0);
    }
    sh.groups[tid] = acc;
    __syncthreads();
    if (tid < width) {
      for (int q = 1; q < groups; ++q) acc += sh.groups[q * width + tid];
      finish(h, unit % (kD / 4), sh.top[h], sh.total[h], acc);
    }
    base += width;
    if (base >= units) break;                      // (uniform)
    __syncthreads();
    width = min(units - base, NT);
    groups = NT / width;
    unit = base + tid % width;
    grp = tid / width;
    issue(grp);
  }
}

// What a row ends as: outputs and log-sum-exp, or a partial for another join.  Four channels of a
// head.
__device__ inline void finish_row(const PagedArgs& a, int64_t head, int c4, float m, float l, v4f o) {
  const bool lost = m == kLowest && l == l;        // every attended score was -infinity (none NaN)
  if (lost) o = (v4f){NAN, NAN, NAN, NAN};
  if (a.seg) {
    Partial* s = a.seg + head;
    reinterpret_cast<v4f*>(s->o)[c4] = o;
    if (c4 == 0) *reinterpret_cast<v4f*>(s) = (v4f){m, l, 0.f, 0.f};
    return;
  }
  const v4f zero = {0.f, 0.f, 0.f, 0.f};
  reinterpret_cast<v4f*>(a.out)[head * (kD / 4) + c4] = l == 0.f ? zero : o / l;
  if (a.lse && c4 == 0) a.lse[head] = l == 0.f || lost ? -INFINITY : (m + log2f(l)) * kLn2;
}

}  // namespace
}  // namespace aatc
