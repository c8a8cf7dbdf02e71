// Attention of a tree of drafted tokens over a paged cache, and the acceptance of one of its paths.
//
// Sequence b has n tokens and m drafts behind them; draft i attends the n tokens, its ancestors and
// itself.  A (sequence, KV head) has m G queries, G the query heads of the KV head: column i G + j is
// head j of draft i.  For column c over its attended tokens t
//   z_t = cap tanh(scale q_c . k_t / cap) - slope (pos_c - pos_t),   o_c = sum_t softmax(z)_t v_t.
//
// One pass with a running maximum and sum, on the tile of paged_tile.h: 32 tokens (16 in float32)
// against groups of 16 columns.  Two kernels:
//   up to 16 columns, bound by the memory as one token's attention is: every wave takes tiles for
//   itself, keys and values go from memory to its registers;
//   more, bound by the matrix cores (P in two or three terms: 1.5 or 2 products for one of a plain
//   attention) and the vector units (exponentials, splitting) about alike: the waves of a workgroup
//   share the tiles of a stage in LDS, each with 16 or 32 of its columns, so that a compute unit reads
//   keys and values once for up to 128 columns.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "drafts.h"
#include "paged_plan.h"
#include "paged_tile.h"
#include "params.h"
#include "wave_scan.h"

namespace aatc {
namespace {

// One workgroup a compute unit, so that a row has few parts to join.
constexpr int kTreeGroups = 256;
// Or four, of the narrow kernel for more rows than these.
constexpr int kFewRows = 128, kSmallGroups = 1024;
constexpr int kGroup = 16;                        // columns of a group
constexpr int kMostCols = 128;                    // of a workgroup
// Runs are a multiple of so many tiles, twice that at least: what a workgroup computes in about the time
// that the join takes.  `slow`: the wide kernel with four waves, one a SIMD.  (648 tokens, 42 columns,
// float32 queries over bf16: 19 us, 28 with the others' 8; 924 float32 tokens, 20 columns: 19 and 28; 2 x
// 600, 371 columns: 38 and 44; 16 x 400, 280 columns: 88 and 90.  It loses where short rows fill the chip
// as they are: 11 x 290 float32 tokens, 371 columns: 65 and 60.)
constexpr int quantum_of(int cols, bool slow) { return slow ? 2 : cols <= 64 ? 8 : 4; }
// Weights are powers of 2 relative to a reference that is renewed when a weight would pass 2^kMost, and
// then so that the highest one is 2^kFirst: sums and outputs are rescaled rarely (when a score rises by
// 2, in f16 6, for any of a wave's columns).  bf16 and float32: weights of at most 1, so that sums stay as
// far from float32's range as those of one token's attention.  (An exponent's own rounding grows with
// it: with 2^-8 in place of 2^-2 outputs were 2.1e-7 off, 1.2e-7 now, and no case took less time.)  f16:
// its values leave room, and small weights stay off the denormals.
template <class M>
constexpr float kMost = std::is_same_v<typename M::Elem, _Float16> ? 15.f : 0.f;
template <class M>
constexpr float kFirst = std::is_same_v<typename M::Elem, _Float16> ? 9.f : -2.f;

// With references from here on (exponents of 2) scores are scaled and rounded before the reference is taken
// off, as on every other path: a fused product keeps bits that the reference, itself rounded, has not.
// They are half a last place of the score: 2^-17 of a weight here, but 2^128 of one from 2^32 on.
constexpr float kLarge = 256.f;

// The window that the shallowest and the deepest of m drafts have together.
__host__ __device__ inline int window_of(int window, int m) {
  return window > 0 ? min(window, 1 << 30) + m - 1 : 0;
}

// Who the columns of a workgroup are, and who descends from whom (LDS).
struct TreeInfo {
  uint64_t family[kMaxDrafts];                     // a draft and its ancestors
  int depth[kMaxDrafts];
  int draft[kMostCols];
  float slope[kMostCols];
};

constexpr int kLaneRows = 256;                    // sequences that lanes of a wave have to themselves

// This thread's number plus those of the threads before it; `total`: of all.
template <int W>
__device__ inline int scan_all(int x, int* space, int& total) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int incl = wave_scan_sum(x);
  __syncthreads();                                 // (the space's last readers are done)
  if (lane == 63) space[wave] = incl;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const int s = space[w];
    incl += w < wave ? s : 0;
    total += s;
  }
  total = __builtin_amdgcn_readfirstlane(total);
  return incl;
}

__device__ inline int cached_of(const TreeArgs& a, int b) {
  return min(max(a.p.seq_len[b], 0), a.p.len_max);
}
__device__ inline int drafts_of(const TreeArgs& a, int b) {
  return a.n_draft ? min(max(a.n_draft[b], 0), a.drafts) : a.drafts;
}

// The runs: every row (a sequence and KV head, all columns) in runs of nearly equal length, the runs
// of all rows in one list.
struct TreeRun {
  int seq, kvh, part, parts;
  int first, last;                                 // tiles
  int shared;                                      // the row's first part slot (part q's: heads q further)
  int len, m;                                      // tokens, drafts
  RowTiles rt;
};

// Run `unit` of the list; false: there is none (for all threads alike).
template <int TT, int W>
__device__ inline bool find_run(const TreeArgs& a, int unit, int (*scan)[W], int* found, TreeRun& r) {
  constexpr int NT = 64 * W;
  const PagedArgs& p = a.p;
  const int tid = threadIdx.x, lane = tid & 63, heads = p.n_kv_heads;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  auto tiles_of = [&](int b) {
    const int m = drafts_of(a, b);
    return row_tiles(cached_of(a, b) + m, window_of(p.window, m), p.sink, TT);
  };
  // Rows that fit the chip are cut into runs that do; more rows into runs as long as the average
  // share: no more than `units` of them beyond one a row.
  auto share = [&](int tiles, int longest, int rows, auto count) {
    return rows * heads <= a.units
               ? a.quantum * smallest_rounds(tiles * heads, longest, rows * heads, a.units, a.quantum, count)
               : max((int)(((int64_t)tiles * heads + a.units - 1) / a.units), kRoundsMin * a.quantum);
  };
  int before = 0, shared = 0, most;
  r.seq = 0;
  if (p.batch == 1) {
    if (drafts_of(a, 0) == 0) return false;
    r.rt = tiles_of(0);
    most = share(r.rt.n, r.rt.n, 1, [&](int q) { return heads * runs_of(r.rt.n, q); });
  } else if (p.batch <= kLaneRows) {
    // Some sequences a lane; every wave does the same.
    constexpr int S = kLaneRows / 64;
    int n_of[S], tiles = 0, rows = 0, longest = 0;
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const int b = lane + 64 * i;
      n_of[i] = b < p.batch && drafts_of(a, b) ? tiles_of(b).n : 0;
      tiles += n_of[i];
      rows += n_of[i] > 0;
      longest = max(longest, n_of[i]);
    }
    tiles = wave_total(tiles);
    if (tiles == 0) return false;
    rows = wave_total(rows);
    longest = __builtin_amdgcn_readlane(wave_scan(longest, 0, [](int x, int y) { return max(x, y); }), 63);
    most = share(tiles, longest, rows, [&](int q) {
      int n = 0;
#pragma unroll
      for (int i = 0; i < S; ++i) n += runs_of(n_of[i], q);
      return heads * wave_total(n);
    });
    int runs = 0, in_shared = 0, owner = -1;       // of the sequences before
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const int k = runs_of(n_of[i], most), mine = heads * k;
      const int incl = runs + wave_scan_sum(mine);
      const int at_shared = in_shared + wave_scan_sum(k > 1 ? mine : 0);
      const uint64_t has = __builtin_amdgcn_ballot_w64(unit >= incl - mine && unit < incl);
      if (has) {                                   // (one lane, of one of the rounds)
        owner = __builtin_ctzll(has);
        r.seq = owner + 64 * i;
        before = __builtin_amdgcn_readlane(incl - mine, owner);
        shared = __builtin_amdgcn_readlane(at_shared - (k > 1 ? mine : 0), owner);
      }
      runs = __builtin_amdgcn_readlane(incl, 63);
      in_shared = __builtin_amdgcn_readlane(at_shared, 63);
    }
    if (owner < 0) return false;
    r.rt = tiles_of(r.seq);
  } else {
    const int each = (p.batch + NT - 1) / NT;
    const int b0 = min(tid * each, p.batch), b1 = min(b0 + each, p.batch);
    int mine = 0, longest = 0, rows = 0, tiles;
    for (int b = b0; b < b1; ++b) {
      const int t = drafts_of(a, b) ? tiles_of(b).n : 0;
      mine += t;
      rows += t > 0;
      longest = max(longest, t);
    }
    scan_all<W>(mine, scan[0], tiles);
    scan_all<W>(rows, scan[1], rows);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) longest = max(longest, __shfl_xor(longest, o, 64));
    __syncthreads();
    if (lane == 0) scan[0][wave] = longest;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) longest = max(longest, scan[0][w]);
    longest = __builtin_amdgcn_readfirstlane(longest);
    if (tiles == 0) return false;
    auto runs = [&](int q) {
      int n = 0, all;
      for (int b = b0; b < b1; ++b) n += drafts_of(a, b) ? runs_of(tiles_of(b).n, q) : 0;
      scan_all<W>(n, scan[0], all);
      return heads * all;
    };
    most = share(tiles, longest, rows, runs);
    // Which sequence has this run, and the runs and the shared rows' runs before it.
    int n = 0, s = 0, total, spare;
    for (int b = b0; b < b1; ++b) {
      const int k = drafts_of(a, b) ? runs_of(tiles_of(b).n, most) : 0;
      n += heads * k;
      s += k > 1 ? heads * k : 0;
    }
    const int incl = scan_all<W>(n, scan[0], total);
    int at_shared = scan_all<W>(s, scan[1], spare) - s;
    if (unit >= total) return false;
    int at = incl - n;
    if (unit >= at && unit < incl) {               // (one thread)
      int b = b0;
      for (;; ++b) {
        const int k = drafts_of(a, b) ? runs_of(tiles_of(b).n, most) : 0;
        if (unit < at + heads * k) break;
        at += heads * k;
        at_shared += k > 1 ? heads * k : 0;
      }
      found[0] = b;
      found[1] = at;
      found[2] = at_shared;
    }
    __syncthreads();
    r.seq = __builtin_amdgcn_readfirstlane(found[0]);
    before = __builtin_amdgcn_readfirstlane(found[1]);
    shared = __builtin_amdgcn_readfirstlane(found[2]);
    r.rt = tiles_of(r.seq);
  }
  r.parts = runs_of(r.rt.n, most);
  r.kvh = (unit - before) % heads;
  r.part = (unit - before) / heads;
  if (r.part >= r.parts) return false;
  r.shared = shared + r.kvh;
  r.len = cached_of(a, r.seq);
  r.m = drafts_of(a, r.seq);
  r.first = run_begin(r.rt.n, r.parts, r.part);
  r.last = run_begin(r.rt.n, r.parts, r.part + 1);
  return true;
}

// Families and depths of a sequence's drafts (one wave, a lane a draft).
__device__ inline void find_families(const TreeArgs& a, const TreeRun& r, TreeInfo& info) {
  const int lane = threadIdx.x & 63;
  int up = lane < r.m ? (a.parent ? a.parent[(int64_t)r.seq * a.drafts + lane] : lane - 1) : -1;
  up = up < lane ? max(up, -1) : -1;
  uint64_t family = (uint64_t)1 << lane;
#pragma unroll
  for (int d = 1; d < kMaxDrafts; d <<= 1) {       // ancestors up to 2 d - 1 steps away
    const int from = max(up, 0);
    const uint64_t theirs = __shfl(family, from, 64);
    const int higher = __shfl(up, from, 64);
    family |= up >= 0 ? theirs : 0;
    up = up >= 0 ? higher : -1;
  }
  info.family[lane] = family;
  info.depth[lane] = __popcll(family) - 1;
}

// Where the tokens of a sequence and KV head lie.
struct TreePages {
  const PagedArgs& p;
  const int32_t* row;
  int64_t head;
  __device__ TreePages(const PagedArgs& args, int seq, int kvh)
      : p(args), row(args.table + seq * args.table_stride), head(kvh * args.head_stride) {}
  __device__ int page_of(int t) const {
    const int i = t >> p.page_shift;
    return i < p.max_pages ? row[i] : -1;
  }
  __device__ bool exists(int page) const { return (page >= 0) & (page < p.n_pages); }
  __device__ int64_t slot_of(int t, int page) const {
    return head + (exists(page) ? page : 0) * p.page_stride +
           (t & ((1 << p.page_shift) - 1)) * p.tok_stride;
  }
};

// What a wave has of C groups of columns, from column col0 of the workgroup's block on: running
// maxima (exponents of 2), sums and value sums (acc[c][j][i]: channel M::channel(j, i, g), or where
// values come turned M::turned_channel(j, i, g), of column 16 c + n).
// TURNED: values come turned from LDS (product j then has other channels).
template <class M, int QT, int C, bool TURNED>
struct TreeWave {
  using Tile = M;
  // A column's value sums, four channels at a time.
  __device__ void store(int c, float* to) const {
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      if constexpr (TURNED) {
        *reinterpret_cast<v4f*>(to + M::turned_channel(x, 0, g)) = acc[c][x];
      } else {                                     // (channels of four products follow each other)
        const int j = x / 4 * 4, i = x % 4;
        *reinterpret_cast<v4f*>(to + M::channel(j, i, g)) =
            (v4f){acc[c][j][i], acc[c][j + 1][i], acc[c][j + 2][i], acc[c][j + 3][i]};
      }
    }
  }
  static constexpr int TT = M::kTokens, NM = M::kMine;
  const PagedArgs& p;
  const TreeInfo& info;
  const int n = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
  int col0, len, end, lo;
  typename M::template Query<QT> q[C];
  v4f acc[C][8];
  float m_run[C], l_run[C];
  unsigned seen = 0u;                              // bit c: any token attended by the lane's column
  bool odd = false;                                // values that are not finite in a masked tile
  bool plain;                                      // scores are only scaled, references below kLarge

  __device__ TreeWave(const TreeArgs& a, const TreeRun& r, TreeInfo& space, int block, int first,
                      int columns)
      : p(a.p), info(space), col0(first), len(r.len), end(r.len + r.m),
        plain(a.p.cap == 0.f && !a.p.slopes && a.p.scale > 0.f) {
    lo = p.window > 0 ? max(0, end - window_of(p.window, r.m)) : 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = first + c * kGroup + n;
      const bool on = col < columns;
      const int x = block * a.block_cols + (on ? col : 0), i = x / p.G, j = x - i * p.G;
      // (columns that are not there are the first one's: a choice would wait for the load)
      q[c].load(p.q, p.q_dtype,
                ((int64_t)r.seq * a.drafts + i) * p.q_stride + (int64_t)(r.kvh * p.G + j) * kD, true, g);
      if (g == 0) {                                // (waves with the same columns write the same)
        space.draft[col] = i;
        space.slope[col] = p.slopes && on ? p.slopes[r.kvh * p.G + j] * kLog2e : 0.f;
      }
      m_run[c] = -INFINITY;
      l_run[c] = 0.f;
#pragma unroll
      for (int j8 = 0; j8 < 8; ++j8) acc[c][j8] = (v4f){0.f, 0.f, 0.f, 0.f};
    }
  }

  // A tile that all columns attend as a whole needs no masks: the deepest draft stands at most at
  // end - 1.  `there`: whether the lane's values' page is.
  __device__ bool is_whole(int t0, bool there) const {
    return t0 + TT <= len &&
           (p.window == 0 || t0 > end - 1 - p.window || t0 + TT <= p.sink) &&
           __builtin_amdgcn_ballot_w64(!there) == 0;
  }

  // Whether any column may attend token t, if its page exists.
  __device__ bool counts(int t) const { return (t < end) & ((t >= lo) | (t < p.sink)); }
  // Tokens that no column attends become zeros; returns which others are not finite (bit e).
  __device__ unsigned mask_values(int t0, bool there, typename M::Values& val) const {
#pragma unroll
    for (int e = 0; e < NM; ++e) val.keep(e, there & counts(t0 + NM * g + e));
    unsigned dirty = 0u;
    if (__builtin_amdgcn_ballot_w64(M::any_bad(val)))
#pragma unroll
      for (int e = 0; e < NM; ++e)
        dirty |= __builtin_amdgcn_ballot_w64(M::bad(val, e)) >> (16 * g) & 0xffffu ? 1u << e : 0u;
    return dirty;
  }

  // Scores as exponents of 2, -infinity where a column does not attend; returns where it does (bit e).
  __device__ unsigned weigh(int c, int t0, bool whole, bool there, float (&z)[NM]) const {
    unsigned bits = ~0u;
    if (p.cap > 0.f) {
      const float in = p.scale / p.cap, out = p.cap * kLog2e;
#pragma unroll
      for (int e = 0; e < NM; ++e) z[e] = out * tanh_of(z[e] * in);
    } else {
#pragma unroll
      for (int e = 0; e < NM; ++e) z[e] *= p.scale * kLog2e;
    }
    if (p.slopes || !whole) {
      const int col = col0 + c * kGroup + n;
      const int draft = info.draft[col], pos = len + info.depth[draft];
      const int first = t0 + NM * g;
      // Positions of the lane's tokens, where they matter.
      auto at = [&](int e) {
        const int j = min(max(first + e - len, 0), kMaxDrafts - 1);
        return first + e < len ? first + e : len + info.depth[j];
      };
      if (p.slopes) {
        const float slope = info.slope[col];
#pragma unroll
        for (int e = 0; e < NM; ++e) z[e] -= slope * (float)(pos - (whole ? first + e : at(e)));
      }
      if (!whole) {
        // Bit e: a token of the sequence, or a draft of the column's family (bits of no draft are 0).
        const uint64_t family = info.family[draft];
        const int j = first - len;
        bits = (unsigned)(j >= 0 ? j < kMaxDrafts ? family >> j : 0
                          : j <= -NM ? ~(uint64_t)0 : family << -j | (((uint64_t)1 << -j) - 1));
        if (p.window)
#pragma unroll
          for (int e = 0; e < NM; ++e)
            if (!((pos - at(e) < p.window) | (first + e < p.sink))) bits &= ~(1u << e);
        bits = there ? bits & ((1u << NM) - 1u) : 0u;
#pragma unroll
        for (int e = 0; e < NM; ++e) z[e] = bits >> e & 1u ? z[e] : -INFINITY;
      }
    }
    return bits;
  }

  // One tile.  next_values and next_keys: called when the registers are free for the next ones.
  template <class V, class K>
  __device__ void step(int t0, bool there, const typename M::Keys& key, typename M::Values& val,
                       V next_values, K next_keys) {
    const bool whole = is_whole(t0, there);
    if (!whole) {
      const unsigned dirty = mask_values(t0, there, val);
      if (__builtin_amdgcn_ballot_w64(dirty != 0u)) {
        odd = true;                                // (these tokens: odd_values)
#pragma unroll
        for (int e = 0; e < NM; ++e) val.keep(e, !(dirty >> e & 1u));
      }
    }
    typename M::Turned turned;
    M::turn(val, turned);
    next_values();
    weigh_and_add(t0, whole, there, key, turned, next_keys);
  }
  __device__ void step(int t0, bool there, const typename M::Keys& key, typename M::Turned& turned) {
    const bool whole = is_whole(t0, there);
    if (!whole) {
      unsigned on = 0u;
#pragma unroll
      for (int e = 0; e < NM; ++e) on |= there & counts(t0 + NM * g + e) ? 1u << e : 0u;
      M::keep_turned(turned, on);
      if (__builtin_amdgcn_ballot_w64(M::any_bad(turned))) {
        odd = true;                                // (these values: odd_values)
        M::drop_bad(turned);
      }
    }
    weigh_and_add(t0, whole, there, key, turned, [] {});
  }

  template <class K>
  __device__ __forceinline__ void weigh_and_add(int t0, bool whole, bool there,
                                                const typename M::Keys& key,
                                                const typename M::Turned& turned, K next_keys) {
    float z[C][NM];
#pragma unroll
    for (int c = 0; c < C; ++c) M::template scores<QT>(key, q[c], z[c]);
    next_keys();
    float unit = p.scale * kLog2e;                 // (scores that are only scaled are so on the way)
    if (whole && plain) {
      seen = ~0u;
    } else {
      unit = 1.f;
#pragma unroll
      for (int c = 0; c < C; ++c) seen |= weigh(c, t0, whole, there, z[c]) ? 1u << c : 0u;
    }
    float top[C];
    bool higher = false;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      top[c] = z[c][0];
#pragma unroll
      for (int e = 1; e < NM; ++e) top[c] = fmaxf(top[c], z[c][e]);
      higher |= top[c] * unit > m_run[c] + kMost<M>;
    }
    if (__builtin_amdgcn_ballot_w64(higher)) {
      bool far = false;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const float most = over_groups_max(top[c]) * unit;
        const float next = most > m_run[c] + kMost<M> ? most - kFirst<M> : m_run[c];
        const float ref = next == -INFINITY ? 0.f : next;
        far |= !(fabsf(ref) < kLarge);
        const float sa = __builtin_amdgcn_exp2f(m_run[c] - ref);    // (0 at the first tile)
        l_run[c] *= sa;
        m_run[c] = next;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[c][j] *= sa;
      }
      if (__builtin_amdgcn_ballot_w64(far)) {
        plain = false;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < NM; ++e) z[c][e] *= unit;
        unit = 1.f;
      }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const float ref = m_run[c] == -INFINITY ? 0.f : m_run[c];
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < NM; ++e) {
        z[c][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[c][e], unit, -ref));
        sum += z[c][e];
      }
      l_run[c] += sum;
      const auto terms = M::split(z[c]);
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[c][j] = M::add(turned, j, terms, acc[c][j]);
    }
  }

  // Values that are not finite count for the columns that attend them and for no others (0 times them
  // is NaN): the tokens of a tile that have such, one by one, with a choice behind the product.
  __device__ void odd_values(int t0, const TreePages& pages) {
    const int vp = pages.page_of(t0 + 8 * M::value_block(g));
    const bool there = pages.exists(vp);
    if (is_whole(t0, there)) return;               // (uniform)
    typename M::Values val;
    val.load(p.v + pages.slot_of(t0 + NM * g, vp), p.tok_stride, n);
    const unsigned dirty = mask_values(t0, there, val);
    if (!__builtin_amdgcn_ballot_w64(dirty != 0u)) return;
    typename M::Keys key;
    key.load(p.k + pages.slot_of(t0 + M::key_token(0, n), pages.page_of(t0 + 8 * M::key_block(n))),
             p.tok_stride, g);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float z[NM];
      M::template scores<QT>(key, q[c], z);
      const unsigned bits = weigh(c, t0, false, there, z);
      const float ref = m_run[c] == -INFINITY ? 0.f : m_run[c];
      for (int tok = 0; tok < TT; ++tok) {
        const int ge = tok / NM, te = tok % NM;
        if (!__builtin_amdgcn_ballot_w64(g == ge && (dirty >> te & 1u))) continue;
        float w[NM];                               // the token in place of the first
        w[0] = z[0];
#pragma unroll
        for (int e = 1; e < NM; ++e) {
          w[0] = e == te ? z[e] : w[0];
          w[e] = 0.f;
        }
        w[0] = __builtin_amdgcn_exp2f(w[0] - ref);
        typename M::Turned turned;
        if constexpr (TURNED) {
          const int t = t0 + tok, page = pages.page_of(t);
          const char* row = p.v + pages.slot_of(t, page) + 2 * n;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint32_t v = *reinterpret_cast<const uint16_t*>(row + 32 * j);
            turned.a[j] = (v4u){g == ge && M::bad16(v) ? v : 0u, 0u, 0u, 0u};   // (the others are in)
          }
        } else {
          typename M::Values one = val;
#pragma unroll
          for (int e = 1; e < NM; ++e) {
            M::take(one, val, e, e == te);
            one.keep(e, false);
          }
          one.keep(0, g == ge);
          M::turn(one, turned);
        }
        const bool on = __shfl(bits, n + 16 * ge, 64) >> te & 1u;
        const auto terms = M::split(w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const v4f sum = M::add(turned, j, terms, acc[c][j]);
#pragma unroll
          for (int x = 0; x < 4; ++x) acc[c][j][x] = on ? sum[x] : acc[c][j][x];
        }
      }
    }
  }
};

// LDS of the joins: the waves' sums of a group each, rows padded for the banks; the (column, part)
// maxima and sums of a row.
constexpr int kSumsFloats = kGroup * (kD + 4);

template <int W>
struct TreeSpace {
  TreeInfo info;
  float m[W][kGroup], l[W][kGroup];
  int scan[2][W], found[4];
};

// Four channels of a column's result.
__device__ inline void finish_column(const TreeArgs& a, const TreeRun& r, int i, int column, int c4,
                                     float top, float total, v4f o) {
  const PagedArgs& p = a.p;
  const int64_t head = ((int64_t)r.seq * a.drafts + i) * p.n_q_heads + r.kvh * p.G + column - i * p.G;
  const bool lost = top == kLowest && total == total;       // attended scores were all -infinity
  if (lost) o = (v4f){NAN, NAN, NAN, NAN};
  const v4f zero = {0.f, 0.f, 0.f, 0.f};
  reinterpret_cast<v4f*>(p.out)[head * (kD / 4) + c4] = total == 0.f ? zero : o / total;
  if (p.lse && c4 == 0)
    p.lse[head] = total == 0.f || lost ? -INFINITY : (top + log2f(total)) * kLn2;
}
// Where part q of the row is, bytes from the workspace's first slot.
__device__ inline int part_at(const TreeArgs& a, const TreeRun& r, int cb, int q, int col) {
  return (((r.shared + q * a.p.n_kv_heads) * a.blocks + cb) * a.block_cols + col) * (int)sizeof(Partial);
}

// What becomes of the waves' sums: waves w TW .. w TW + TW - 1 have the same columns (C groups from
// w 16 C on) and different tokens.  sums(wave): kSumsFloats of LDS.
template <int W, int TW, class Wave, class Sums, int C>
__device__ __forceinline__ void finish_run(const TreeArgs& a, const TreeRun& r, int cb, int columns,
                                           TreeSpace<W>& sh, Wave& x, Sums sums,
                                           std::integral_constant<int, C>) {
  constexpr int NT = 64 * W, CW = W / TW;
  const PagedArgs& p = a.p;
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    __syncthreads();                               // the tiles, or the last group's sums, are read
    const float l = over_groups_sum(x.l_run[c]);
    unsigned any = x.seen >> c & 1u;
    any |= __shfl_xor(any, 16, 64);
    any |= __shfl_xor(any, 32, 64);
    // (NaN scores: the sum is NaN)
    const bool low = any && x.m_run[c] == -INFINITY && l == 0.f;
    if (g == 0) {
      sh.m[wave][n] = low ? kLowest : x.m_run[c];
      sh.l[wave][n] = low ? 1.f : l;
    }
    x.store(c, sums(wave) + n * (kD + 4));
    __syncthreads();
    for (int y = tid; y < CW * kGroup * (kD / 4); y += NT) {
      const int h = y / (kD / 4) % kGroup, c4 = y % (kD / 4), w0 = y / (kGroup * (kD / 4)) * TW;
      const int col = (w0 / TW * C + c) * kGroup + h;
      float mm = sh.m[w0][h];
#pragma unroll
      for (int w = 1; w < TW; ++w) mm = fmaxf(mm, sh.m[w0 + w][h]);
      float ll = 0.f;
      v4f o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < TW; ++w) {
        const float m = sh.m[w0 + w][h], lw = sh.l[w0 + w][h];
        const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mm);
        ll += lw == 0.f ? 0.f : f * lw;
        o += f * *reinterpret_cast<const v4f*>(sums(w0 + w) + h * (kD + 4) + 4 * c4);
      }
      if (col >= columns) continue;
      if (r.parts == 1) {
        finish_column(a, r, sh.info.draft[col], cb * a.block_cols + col, c4, mm, ll, o);
      } else {
        v4f* slot = reinterpret_cast<v4f*>(reinterpret_cast<char*>(a.p.parts) +
                                           part_at(a, r, cb, r.part, col));
        slot[1 + c4] = o;
        if (c4 == 0) slot[0] = (v4f){mm, ll, 0.f, 0.f};
      }
    }
  }
}

// The parts of the rows that are shared, joined in their order: the same grid as the runs', and as many
// workgroups as a row has parts take a share of its columns each.  (A join by the last of a row's
// workgroups would read up to 4 MiB alone: 32 parts of 256 columns took 100 us.)  Latency bounds it: the
// plan, then the parts' maxima, then their sums, of which up to eight threads take a share (64 drafts of
// 32768 tokens: 5.0 us, 7.1 with one thread for all parts).  Rows of one group have little to join: two
// waves (384 rows in three parts: 9.8 us, 12 with eight waves).
template <int TT, int W>
__global__ __launch_bounds__(64 * W) void tree_join_kernel(TreeArgs a) {
  constexpr int NT = 64 * W;
  constexpr int kPairs = kMostCols + kSmallGroups;  // columns / parts of them, for each part
  __shared__ int scan[2][W], found[4];
  __shared__ float weight[kPairs], sum[kPairs], top[kMostCols], total[kMostCols];
  __shared__ v4f shares[NT];
  const PagedArgs& p = a.p;
  const int tid = threadIdx.x, block = (int)blockIdx.x;
  const int unit = (block >> 3) / a.blocks * 8 + (block & 7), cb = (block >> 3) % a.blocks;
  TreeRun r;
  if (!find_run<TT, W>(a, unit, scan, found, r) || r.parts == 1) return;
  const int columns = min(r.m * p.G - cb * a.block_cols, a.block_cols), parts = r.parts;
  if (columns <= 0) return;
  const int first = columns * r.part / parts, count = columns * (r.part + 1) / parts - first;
  const char* slots = reinterpret_cast<const char*>(p.parts);
  auto slot = [&](int q, int col, int off) {
    return *reinterpret_cast<const v4f*>(slots + part_at(a, r, cb, q, first + col) + off);
  };
  constexpr int U = 8;                             // parts in flight, the first before their weights
  v4f v[U];
  auto fetch = [&](int y, int q0) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      v[u] = slot(min(q0 + u, parts - 1), min(y / (kD / 4), count - 1), 16 + 16 * (y % (kD / 4)));
  };
  // Four channels a thread; where that leaves threads without any, up to eight share the parts.
  const int items = count * (kD / 4);
  const int split = count == 0 || 2 * items > NT ? 1 : 4 * items > NT ? 2 : 8 * items > NT ? 4 : 8;
  const int per = (parts + split - 1) / split, mine = split > 1 ? tid / items : 0;
  const int y0 = tid - mine * items, q_first = mine * per, q_last = min(q_first + per, parts);
  if (count > 0 && mine < split) fetch(y0, q_first);
  for (int y = tid; y < count * parts; y += NT) {
    const v4f ml = slot(y % parts, y / parts, 0);
    weight[y] = ml[0];
    sum[y] = ml[1];
  }
  __syncthreads();
  for (int col = tid >> 3; col < count; col += NT / 8) {           // eight threads a column
    float m = -INFINITY, l = 0.f;
    for (int q = tid & 7; q < parts; q += 8)
      if (sum[col * parts + q] != 0.f) m = fmaxf(m, weight[col * parts + q]);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    const float ref = m == -INFINITY ? 0.f : m;
    for (int q = tid & 7; q < parts; q += 8) {
      const float s = sum[col * parts + q];
      const float w = s == 0.f ? 0.f : __builtin_amdgcn_exp2f(weight[col * parts + q] - ref);
      l += s == 0.f ? 0.f : w * s;                 // (NaN stays)
      weight[col * parts + q] = w;
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) l += __shfl_xor(l, o, 64);
    if ((tid & 7) == 0) {
      top[col] = m;
      total[col] = l;
    }
  }
  __syncthreads();
  auto joined = [&](int y) {
    v4f o = {0.f, 0.f, 0.f, 0.f};
    for (int q0 = q_first; q0 < q_last; q0 += U) {
      if (q0 > q_first || y != y0) fetch(y, q0);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float w = q0 + u < q_last ? weight[y / (kD / 4) * parts + q0 + u] : 0.f;
        if (w != 0.f) o += w * v[u];
      }
    }
    return o;
  };
  auto finish = [&](int y, v4f o) {
    const int col = y / (kD / 4), column = cb * a.block_cols + first + col;
    finish_column(a, r, column / p.G, column, y % (kD / 4), top[col], total[col], o);
  };
  if (split == 1) {
    for (int y = tid; y < items; y += NT) finish(y, joined(y));
    return;
  }
  if (mine < split) shares[tid] = joined(y0);
  __syncthreads();
  if (mine > 0) return;
  v4f o = shares[tid];
  for (int x = 1; x < split; ++x) o += shares[x * items + tid];
  finish(tid, o);
}

// Up to 16 columns: every wave has tiles of its own; keys and values one tile ahead, pages two.  Few rows:
// eight waves a workgroup, so that a row has few parts to join.  Many: four, four times as many workgroups,
// whose runs are dealt more evenly (384 rows of 129 float32 tiles: 145 us with the join, 172 with eight).
template <class M, int QT, int W>
__global__ __launch_bounds__(64 * W, 2) void tree_narrow_kernel(TreeArgs a) {
  constexpr int TT = M::kTokens, NM = M::kMine;
  __shared__ TreeSpace<W> sh;
  __shared__ __align__(16) float space[W * kSumsFloats];
  const PagedArgs& p = a.p;
  const int n = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  TreeRun r;
  if (!find_run<TT, W>(a, (int)blockIdx.x, sh.scan, sh.found, r)) return;
  const int columns = r.m * p.G;
  const TreePages pages(p, r.seq, r.kvh);
  TreeWave<M, QT, 1, false> x(a, r, sh.info, 0, 0, columns);
  typename M::Keys key;
  typename M::Values val;
  auto load_keys = [&](int t0, int page) {
    key.load(p.k + pages.slot_of(t0 + M::key_token(0, n), page), p.tok_stride, g);
  };
  auto load_values = [&](int t0, int page) {
    val.load(p.v + pages.slot_of(t0 + NM * g, page), p.tok_stride, n);
  };
  auto key_page = [&](int t0) { return pages.page_of(t0 + 8 * M::key_block(n)); };
  auto value_page = [&](int t0) { return pages.page_of(t0 + 8 * M::value_block(g)); };
  const int begin = r.first + wave, last = r.last;
  int t0 = r.rt.token(min(begin, last - 1), TT), t1 = r.rt.token(min(begin + W, last - 1), TT);
  int vp = value_page(t0), kp1 = key_page(t1), vp1 = value_page(t1);
  if (begin < last) {
    load_keys(t0, key_page(t0));
    load_values(t0, vp);
  }
  if (wave == W - 1) find_families(a, r, sh.info);
  __syncthreads();
  for (int i = begin; i < last; i += W) {
    const bool more = i + W < last;
    const int t2 = r.rt.token(min(i + 2 * W, last - 1), TT);
    int kp2, vp2;
    x.step(t0, pages.exists(vp), key, val,
           [&] { if (more) load_values(t1, vp1); },
           [&] {
             if (more) load_keys(t1, kp1);
             kp2 = key_page(t2), vp2 = value_page(t2);
           });
    t0 = t1, vp = vp1;
    t1 = t2, kp1 = kp2, vp1 = vp2;
  }
  if (x.odd)
    for (int i = begin; i < last; i += W) x.odd_values(r.rt.token(i, TT), pages);
  finish_run<W, W>(a, r, 0, columns, sh, x, [&](int w) { return space + w * kSumsFloats; },
                   std::integral_constant<int, 1>{});
}

// More columns: eight waves a workgroup, two a SIMD, or four where registers leave room for one.  A stage has
// kStage tiles, each 8 KiB of keys and 8 KiB of values, loaded straight into LDS, kRing - 1 stages ahead of
// the one that is computed.  Wave w has 16 C columns from
// (w / TW) 16 C on and every TW-th tile.
constexpr int kRingTiles = 8;
constexpr int kStreamed = 2;                       // cache policy nt
constexpr int kValueRing = kRingTiles * 8192;      // the values' place in the ring, behind all keys
// Waits until no more than n vector loads are outstanding, and for LDS.
template <int N>
__device__ inline void wait_loads() {
  static_assert(N < 64, "six bits");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (N >> 4 << 14));
}

// The keys and values of a tile in LDS.  (In assembly, with the wait: the compiler would wait for the
// loads of the next stage too, which go elsewhere in the same array.)
template <class M>
__device__ inline void read_keys(typename M::Keys& to, uint32_t at) {
  v4u x[8];
  static_assert(sizeof to == sizeof x, "eight pieces");
  const uint32_t p[4] = {at, at ^ 64u, at ^ 128u, at ^ 192u};
  asm volatile(
      "ds_read_b128 %0, %8 offset:%16\n\tds_read_b128 %1, %9 offset:%17\n\t"
      "ds_read_b128 %2, %10 offset:%18\n\tds_read_b128 %3, %11 offset:%19\n\t"
      "ds_read_b128 %4, %12 offset:%20\n\tds_read_b128 %5, %13 offset:%21\n\t"
      "ds_read_b128 %6, %14 offset:%22\n\tds_read_b128 %7, %15 offset:%23\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]),
        "=&v"(x[7])
      : "v"(p[M::key_flip(0)]), "v"(p[M::key_flip(1)]), "v"(p[M::key_flip(2)]),
        "v"(p[M::key_flip(3)]), "v"(p[M::key_flip(4)]), "v"(p[M::key_flip(5)]),
        "v"(p[M::key_flip(6)]), "v"(p[M::key_flip(7)]), "n"(M::key_offset(0)),
        "n"(M::key_offset(1)), "n"(M::key_offset(2)), "n"(M::key_offset(3)), "n"(M::key_offset(4)),
        "n"(M::key_offset(5)), "n"(M::key_offset(6)), "n"(M::key_offset(7))
      : "memory");
  __builtin_memcpy(&to, x, sizeof x);
}
template <class M>
__device__ inline void read_values(typename M::Values& to, uint32_t at) {
  v4u x[8];
  static_assert(sizeof to == sizeof x, "eight pieces");
  const uint32_t p[4] = {at, at ^ 16u, at ^ 32u, at ^ 48u};
  asm volatile(
      "ds_read_b128 %0, %8 offset:%16\n\tds_read_b128 %1, %9 offset:%17\n\t"
      "ds_read_b128 %2, %10 offset:%18\n\tds_read_b128 %3, %11 offset:%19\n\t"
      "ds_read_b128 %4, %12 offset:%20\n\tds_read_b128 %5, %13 offset:%21\n\t"
      "ds_read_b128 %6, %14 offset:%22\n\tds_read_b128 %7, %15 offset:%23\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]),
        "=&v"(x[7])
      : "v"(p[M::value_flip(0)]), "v"(p[M::value_flip(1)]), "v"(p[M::value_flip(2)]),
        "v"(p[M::value_flip(3)]), "v"(p[M::value_flip(4)]), "v"(p[M::value_flip(5)]),
        "v"(p[M::value_flip(6)]), "v"(p[M::value_flip(7)]), "n"(M::value_offset(0)),
        "n"(M::value_offset(1)), "n"(M::value_offset(2)),
        "n"(M::value_offset(3)), "n"(M::value_offset(4)),
        "n"(M::value_offset(5)), "n"(M::value_offset(6)),
        "n"(M::value_offset(7))
      : "memory");
  __builtin_memcpy(&to, x, sizeof x);
}
template <class M>
__device__ inline void read_turned(typename M::Turned& to, uint32_t at) {
  typedef uint32_t v2u __attribute__((ext_vector_type(2)));
  v2u x[8][2];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %16 offset:%24\n\tds_read_b64_tr_b16 %1, %16 offset:%25\n\t"
      "ds_read_b64_tr_b16 %2, %17 offset:%24\n\tds_read_b64_tr_b16 %3, %17 offset:%25\n\t"
      "ds_read_b64_tr_b16 %4, %18 offset:%24\n\tds_read_b64_tr_b16 %5, %18 offset:%25\n\t"
      "ds_read_b64_tr_b16 %6, %19 offset:%24\n\tds_read_b64_tr_b16 %7, %19 offset:%25\n\t"
      "ds_read_b64_tr_b16 %8, %20 offset:%24\n\tds_read_b64_tr_b16 %9, %20 offset:%25\n\t"
      "ds_read_b64_tr_b16 %10, %21 offset:%24\n\tds_read_b64_tr_b16 %11, %21 offset:%25\n\t"
      "ds_read_b64_tr_b16 %12, %22 offset:%24\n\tds_read_b64_tr_b16 %13, %22 offset:%25\n\t"
      "ds_read_b64_tr_b16 %14, %23 offset:%24\n\tds_read_b64_tr_b16 %15, %23 offset:%25\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[2][0]),
        "=&v"(x[2][1]), "=&v"(x[3][0]), "=&v"(x[3][1]), "=&v"(x[4][0]), "=&v"(x[4][1]),
        "=&v"(x[5][0]), "=&v"(x[5][1]), "=&v"(x[6][0]), "=&v"(x[6][1]), "=&v"(x[7][0]),
        "=&v"(x[7][1])
      : "v"(at), "v"(at ^ 32u), "v"(at ^ 64u), "v"(at ^ 96u), "v"(at ^ 128u), "v"(at ^ 160u),
        "v"(at ^ 192u), "v"(at ^ 224u), "n"(0), "n"(4 * M::kRow)
      : "memory");
#pragma unroll
  for (int j = 0; j < 8; ++j) to.a[j] = (v4u){x[j][0][0], x[j][0][1], x[j][1][0], x[j][1][1]};
}

template <class M, int QT, int C, int CW, int W, int kStage>
__global__ __launch_bounds__(64 * W, W / 4) void tree_wide_kernel(TreeArgs a) {
  constexpr int TT = M::kTokens, NM = M::kMine, TW = W / CW;
  constexpr int kRow = M::kRow;
  constexpr int kRing = kRingTiles / kStage;
  constexpr int PT = kStage * TT / W;              // tokens of a stage that a wave loads
  constexpr int kPer = 1024 / kRow;                // tokens of one load of the wave
  static_assert(TW >= 1 && TW <= kStage && 16 * C * CW <= kMostCols, "a tile for every wave");
  __shared__ TreeSpace<W> sh;
  __shared__ __align__(1024) char ring[2 * kValueRing];
  __shared__ int there[kRing][kStage * TT / 8];    // whether the page of 8 tokens is
  const PagedArgs& p = a.p;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // The column blocks of one run read the same tokens: they are on one XCD (workgroups go to the
  // eight in turn) at one time, and meet in its L2.
  const int block = (int)blockIdx.x;
  const int unit = (block >> 3) / a.blocks * 8 + (block & 7), cb = (block >> 3) % a.blocks;
  TreeRun r;
  if (!find_run<TT, W>(a, unit, sh.scan, sh.found, r)) return;
  const int columns = min(r.m * p.G - cb * a.block_cols, a.block_cols);
  if (columns <= 0) return;                        // (uniform)
  const TreePages pages(p, r.seq, r.kvh);
  // (queries first: their wait would be one for all loads before them)
  const int cw = wave / TW, tw = wave % TW;
  TreeWave<M, QT, C, M::kReadsTurned> x(a, r, sh.info, cb, cw * C * kGroup, columns);

  // This wave's PT tokens of a stage: their first one, pages a stage ahead of the loads, and those.
  // (Pages by scalar loads: a vector load's wait would be one for all loads before it.  Every stage has
  // as many loads, so that they can be counted; behind the last tile it is that one again.)
  const int tile = wave * PT / TT, within = wave * PT % TT;
  const auto row = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)pages.row;
  auto token_of = [&](int s) {
    return r.rt.token(min(r.first + s * kStage + tile, r.last - 1), TT) + within;
  };
  auto fetch_pages = [&](int s, int(&page)[PT / 8]) {
    const int t = token_of(s);
#pragma unroll
    for (int b = 0; b < PT / 8; ++b) {
      const int i = __builtin_amdgcn_readfirstlane((t + 8 * b) >> p.page_shift);
      page[b] = i < p.max_pages ? row[i] : -1;
    }
  };
  constexpr int kLoads = 2 * PT / kPer;            // of a stage, of a wave
  auto issue = [&](int s, const int(&page)[PT / 8]) {
    const int t = token_of(s), slot = s % kRing;
#pragma unroll
    for (int i = 0; i < PT / kPer; ++i) {
      const int at = i * kPer + lane / (kRow / 16), c = lane % (kRow / 16);
      const int64_t from = pages.slot_of(t + at, page[i * kPer / 8]) +
                           16 * (c ^ M::turn_of((wave * PT + at) % TT));
      char* to = ring + slot * (kStage * 8192) + (wave * PT + i * kPer) * kRow;
      using Global = const __attribute__((address_space(1))) void*;
      using Local = __attribute__((address_space(3))) void*;
      if (a.far) {                                 // (uniform)
        __builtin_amdgcn_global_load_lds((Global)(p.k + from), (Local)to, 16, 0, kStreamed);
        __builtin_amdgcn_global_load_lds((Global)(p.v + from), (Local)(to + kValueRing), 16, 0, kStreamed);
      } else {
        __builtin_amdgcn_global_load_lds((Global)(p.k + from), (Local)to, 16, 0, 0);
        __builtin_amdgcn_global_load_lds((Global)(p.v + from), (Local)(to + kValueRing), 16, 0, 0);
      }
    }
    if (lane < PT / 8) {
      int on = 0;
#pragma unroll
      for (int b = 0; b < PT / 8; ++b) on = lane == b ? pages.exists(page[b]) : on;
      there[slot][wave * PT / 8 + lane] = on;
    }
  };

  const int stages = (r.last - r.first + kStage - 1) / kStage;
  int page[kRing][PT / 8];
#pragma unroll
  for (int s = 0; s < kRing; ++s) fetch_pages(s, page[s]);
#pragma unroll
  for (int s = 0; s < kRing - 1; ++s) issue(s, page[s]);
  if (wave == W - 1) find_families(a, r, sh.info);
  const bool busy = cw * C * kGroup < columns;     // (uniform)
  // Where the lane's pieces of a tile are (a ring aligned to more than a row: pieces differ in bits of
  // the address).
  const uint32_t key0 = M::key_place(n, g), value0 = M::value_place(n, g);
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)ring;
#pragma unroll 1
  for (int s = 0; s < stages; ++s) {
    wait_loads<(kRing - 2) * kLoads>();            // this wave's part of the stage has come
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();                  // everyone's has, and the stage before is read
    asm volatile("" ::: "memory");
    issue(s + kRing - 1, page[kRing - 1]);
    fetch_pages(s + kRing, page[kRing - 1]);
    const int slot = s % kRing;
    if (busy)
#pragma unroll 1
      for (int k = tw; k < kStage; k += TW) {
        const int i = r.first + s * kStage + k;
        if (i >= r.last) break;                    // (uniform)
        typename M::Keys key;
        const uint32_t from = base + slot * (kStage * 8192) + k * (TT * kRow);
        read_keys<M>(key, from + key0);
        const int t0 = r.rt.token(i, TT);
        const bool on = there[slot][k * TT / 8 + M::value_block(g)] != 0;
        if constexpr (M::kReadsTurned) {
          typename M::Turned turned;
          read_turned<M>(turned, from + kValueRing + value0);
          x.step(t0, on, key, turned);
        } else {
          typename M::Values val;
          read_values<M>(val, from + kValueRing + value0);
          x.step(t0, on, key, val, [] {}, [] {});
        }
      }
  }
  wait_loads<0>();                                 // (the loads behind the last stage)
  if (x.odd)
    for (int i = r.first + tw; i < r.last; i += TW) x.odd_values(r.rt.token(i, TT), pages);
  finish_run<W, TW>(a, r, cb, columns, sh, x,
                    [&](int w) { return reinterpret_cast<float*>(ring) + w * kSumsFloats; },
                    std::integral_constant<int, C>{});
}

// A (sequence, KV head)'s columns in blocks of 32, 64 or 128, the smallest that hold an even share; the
// first are full, the last has the rest.  A block's groups are dealt to `cw` sets of waves, c groups each.
// (Blocks of 256 columns, which read keys and values half as often but have twice the parts to join, took
// as long for 64 drafts of 32768 tokens and longer for fewer tokens: 28.3 us at 1000 tokens, 33.7.)
struct Blocks {
  int blocks, c, cw;
  int cols() const { return c * cw * kGroup; }
};
Blocks blocks_of(int drafts, int G) {
  const int groups = (drafts * G + kGroup - 1) / kGroup;
  if (groups == 1) return {1, 1, 1};
  const int blocks = (groups + 7) / 8, each = (groups + blocks - 1) / blocks;
  return {blocks, each <= 2 ? 1 : 2, each <= 4 ? 2 : 4};
}
bool small_groups(const Blocks& b, int64_t rows) { return b.cols() == kGroup && rows > kFewRows; }
int units_of(const Blocks& b, int64_t rows) {
  return small_groups(b, rows) ? kSmallGroups : std::max(1, kTreeGroups / b.blocks);
}

// Part slots: runs that fit the chip, or at most twice as many where more rows than those are cut.
size_t tree_parts_bytes(const Blocks& b, int64_t rows) {
  const int units = units_of(b, rows);
  return (size_t)(rows <= units ? 1 : 2) * units * b.blocks * b.cols() * sizeof(Partial);
}

}  // namespace

size_t tree_workspace_bytes(int batch, int drafts, int n_q_heads, int n_kv_heads) {
  return tree_parts_bytes(blocks_of(drafts, n_q_heads / n_kv_heads), (int64_t)batch * n_kv_heads);
}

bool tree_fits(int64_t batch, int drafts, int n_q_heads, int n_kv_heads) {
  const int64_t columns = (int64_t)drafts * (n_q_heads / n_kv_heads);
  if (columns > kMaxColumns) return false;
  const Blocks b = blocks_of(drafts, n_q_heads / n_kv_heads);
  return (batch * n_kv_heads + kSmallGroups + 8) * b.blocks <= kMaxTreeGroups;
}

aatc_status launch_tree(TreeArgs a, aatc_dtype c_dtype, void* workspace, void* stream) {
  const bool same = a.p.q_dtype == (int)c_dtype, full = c_dtype == AATC_F32;
  const Blocks b = blocks_of(a.drafts, a.p.G);
  const int rows = a.p.batch * a.p.n_kv_heads;
  a.blocks = b.blocks;
  a.block_cols = b.cols();
  a.units = units_of(b, rows);
  a.quantum = quantum_of(b.cols(), b.cols() > kGroup && (full || !same));
  a.p.parts = static_cast<Partial*>(workspace);
  const int64_t most = rows <= a.units ? a.units : (int64_t)rows + a.units;
  const int64_t grid = (most + 7) / 8 * 8 * b.blocks;
  const hipStream_t st = (hipStream_t)stream;
  auto launch = [&](auto kernel, int waves) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * waves), 0, st, a);
    return hipGetLastError() == hipSuccess ? AATC_OK : AATC_E_DEVICE;
  };
  using One = std::integral_constant<int, 1>;
  using Three = std::integral_constant<int, 3>;
  auto launch_narrow = [&](auto near, auto past, auto qt) {
    constexpr int QT = decltype(qt)::value;
    if (small_groups(b, rows))
      return a.far ? launch(tree_narrow_kernel<decltype(past), QT, 4>, 4)
                   : launch(tree_narrow_kernel<decltype(near), QT, 4>, 4);
    return a.far ? launch(tree_narrow_kernel<decltype(past), QT, 8>, 8)
                 : launch(tree_narrow_kernel<decltype(near), QT, 8>, 8);
  };
  auto launch_wide = [&](auto m, auto qt) {
    using M = decltype(m);
    constexpr int QT = decltype(qt)::value;
    // Queries of one 16-bit term leave room for two waves a SIMD.
    constexpr int W = QT == 1 && sizeof(typename M::Elem) == 2 ? 8 : 4, S = W == 8 ? 4 : 2;
    if (b.cw == 2)
      return b.c == 1 ? launch(tree_wide_kernel<M, QT, 1, 2, W, S>, W)
                      : launch(tree_wide_kernel<M, QT, 2, 2, W, S>, W);
    return launch(tree_wide_kernel<M, QT, 2, 4, W, 2>, W);
  };
  auto launch_as = [&](auto near, auto past, auto qt) {
    return b.cols() == kGroup ? launch_narrow(near, past, qt) : launch_wide(near, qt);
  };
  auto launch_type = [&](auto near, auto past) {
    return same ? launch_as(near, past, One{}) : launch_as(near, past, Three{});
  };
  a.far = pools_far(a.p, c_dtype);
  const aatc_status e =
      full ? launch_as(Full32<false>{}, Full32<true>{}, One{})
      : c_dtype == AATC_BF16 ? launch_type(Half16<__bf16, false>{}, Half16<__bf16, true>{})
                             : launch_type(Half16<_Float16, false>{}, Half16<_Float16, true>{});
  // (a table that holds no more than a shortest run's tokens has no shared rows)
  const int tt = full ? Full32<false>::kTokens : Half16<__bf16, false>::kTokens;
  if (e != AATC_OK || (a.p.len_max + a.drafts) / tt < kRoundsMin * a.quantum) return e;
  if (small_groups(b, rows))
    return full ? launch(tree_join_kernel<Full32<false>::kTokens, 2>, 2)
                : launch(tree_join_kernel<Half16<__bf16, false>::kTokens, 2>, 2);
  return full ? launch(tree_join_kernel<Full32<false>::kTokens, 8>, 8)
              : launch(tree_join_kernel<Half16<__bf16, false>::kTokens, 8>, 8);
}

namespace {

// Every workgroup of a sequence walks its tree by itself (a wave, a lane a draft: a few steps of a
// ballot each); each of its threads then moves 16 bytes of a head's token, for all of the path's
// tokens: reads go before the writes of the same slots because the path ascends.
__global__ __launch_bounds__(256) void accept_kernel(AcceptArgs a) {
  const int seq = blockIdx.y, lane = threadIdx.x & 63;
  const int len = min(max(a.seq_len[seq], 0), a.len_max);
  const int m = a.n_draft ? min(max(a.n_draft[seq], 0), a.drafts) : a.drafts;
  const int64_t at = (int64_t)seq * a.drafts;
  const bool there = lane < m;
  int up = there ? (a.parent ? a.parent[at + lane] : lane - 1) : -1;
  up = up < lane ? up : -1;
  const int token = there ? a.drafted[at + lane] : 0, choice = there ? a.chosen[at + lane] : -1;
  uint64_t path = m > 0 ? 1u : 0u;
  int now = 0;
  for (;;) {                                       // (`now` grows: at most 63 steps)
    const int want = __builtin_amdgcn_readlane(choice, now);
    const uint64_t next = __builtin_amdgcn_ballot_w64(there & (lane > now) & (up == now) & (token == want));
    if (!next) break;
    now = __builtin_ctzll(next);
    path |= (uint64_t)1 << now;
  }
  const int count = __popcll(path);
  if (blockIdx.x == 0 && threadIdx.x < 64) {
    if (path >> lane & 1) a.path[at + __popcll(path & (((uint64_t)1 << lane) - 1))] = lane;
    if (lane >= count && lane < a.drafts) a.path[at + lane] = -1;
    if (lane == now) {
      a.accepted[seq] = count;
      a.next[seq] = m > 0 ? choice : -1;
      a.len_out[seq] = len + count;
    }
  }

  // Slots that stay need no move.
  if (path == ~(uint64_t)0) return;
  const int stay = __builtin_ctzll(~path);
  if (count == stay) return;
  const int per_layer = 2 * a.n_kv_heads * a.pieces;
  const int64_t x = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (x >= (int64_t)a.layers * per_layer) return;
  const int layer = (int)(x / per_layer), y = (int)(x - (int64_t)layer * per_layer);
  const int piece = y % a.pieces, head = y / a.pieces % a.n_kv_heads;
  char* pool = (y >= a.n_kv_heads * a.pieces ? a.v : a.k) + layer * a.layer_stride +
               head * a.head_stride + 16 * piece;
  const int32_t* row = a.table + seq * a.table_stride;
  auto slot = [&](int t, bool& ok) {
    const int i = t >> a.page_shift;
    const int page = i < a.max_pages ? row[i] : -1;
    ok = (page >= 0) & (page < a.n_pages);
    return pool + (ok ? page : 0) * a.page_stride + (t & ((1 << a.page_shift) - 1)) * a.tok_stride;
  };
  uint64_t rest = path & ~(((uint64_t)1 << stay) - 1);
  for (int to = stay; rest;) {
    constexpr int U = 4;                           // tokens in flight
    v4u data[U];
    char* dst[U];
    bool ok[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int from = rest ? __builtin_ctzll(rest) : 0;
      bool have, goes;
      const char* src = slot(len + from, have);
      dst[u] = slot(len + to + u, goes);
      ok[u] = (rest != 0) & have & goes;
      if (ok[u]) data[u] = *reinterpret_cast<const v4u*>(src);
      rest &= rest - 1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (ok[u]) *reinterpret_cast<v4u*>(dst[u]) = data[u];
    to += U;
  }
}

}  // namespace

aatc_status launch_tree_accept(const AcceptArgs& a, void* stream) {
  const int64_t pieces = (int64_t)a.layers * 2 * a.n_kv_heads * a.pieces;
  const int64_t groups = (pieces + 255) / 256;     // (2^23 at most)
  constexpr int kMost = 65535;                     // sequences of a launch
  for (int b = 0; b < a.batch; b += kMost) {
    AcceptArgs s = a;
    const int64_t at = (int64_t)b * a.drafts;
    s.table += b * a.table_stride;
    s.seq_len += b;
    s.n_draft = a.n_draft ? a.n_draft + b : nullptr;
    s.parent = a.parent ? a.parent + at : nullptr;
    s.drafted += at;
    s.chosen += at;
    s.path += at;
    s.accepted += b;
    s.next += b;
    s.len_out += b;
    const int rows = std::min(a.batch - b, kMost);
    hipLaunchKernelGGL(accept_kernel, dim3((unsigned)groups, (unsigned)rows), dim3(256), 0,
                       (hipStream_t)stream, s);
    if (hipGetLastError() != hipSuccess) return AATC_E_DEVICE;
  }
  return AATC_OK;
}

}  // namespace aatc
