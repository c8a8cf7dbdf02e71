// Attention of a tree of drafted tokens over a paged cache, and the acceptance of one of its paths.
//
// Sequence b has n tokens and m drafts behind them; draft i attends the n tokens, its ancestors and
// itself.  A (sequence, KV head) has m G queries, G the query heads of the KV head: column i G + j is
// head j of draft i.  For column c over its attended tokens t
//   z_t = cap tanh(scale q_c . k_t / cap) - slope (pos_c - pos_t),   o_c = sum_t softmax(z)_t v_t.
//
// One pass with a running maximum and sum, on the tile of paged_tile.h: a wave takes 32 tokens (16 in
// float32) against up to C groups of 16 columns, so that keys and values are read once for all of
// them and values are turned once.  The queries of C > 1 groups lie in LDS as matrix operands.
//
// What bounds it: few columns (m G <= 16) the memory, as one token does; 64 columns and more the
// matrix cores (P in two or three terms: 1.5 or 2 products for one of a plain attention) and the
// vector units (exponentials, splitting) about alike.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "drafts.h"
#include "paged_plan.h"
#include "paged_tile.h"
#include "params.h"

namespace aatc {
namespace {

// Eight waves a workgroup, one workgroup a compute unit: a row has few parts to join.
constexpr int kTreeWaves = 8, kTreeGroups = 256;
constexpr int kGroup = 16;                        // columns of a group
constexpr int kMostGroups = 4;                    // of a workgroup
// The workspace: arrival counters of the rows that are shared (256 bytes apart, left at zero), then
// part slots.  At most twice as many runs as fill the chip belong to shared rows.
constexpr int kTreeSlots = 2 * kTreeGroups, kTreeCounterStride = 64;
constexpr size_t kTreeCountersBytes = (size_t)kTreeSlots * kTreeCounterStride * sizeof(unsigned);
// (column, part) pairs of a joined block: their weights are kept in LDS.
constexpr int kMostPairs = 8192;
// The maximum that weights refer to is renewed when a score passes it by this much (exponents of 2):
// sums and outputs are rescaled rarely.  Weights of 2^(slack + lower) have to fit their type.
template <class M>
constexpr float kSlack = std::is_same_v<typename M::Elem, _Float16> ? 6.f : 8.f;
template <class M>
constexpr float kBelow = std::is_same_v<typename M::Elem, _Float16> ? 9.f : 0.f;

__host__ __device__ inline int window_of(int window, int m) {
  return window > 0 ? min(window, 1 << 30) + m - 1 : 0;
}

template <class M, int QT, int C>
struct TreeSpace {
  using Query = typename M::template Query<QT>;
  static constexpr int kPieces = sizeof(Query::t) / 16;
  union {
    v4u q[C][kPieces][64];
    float sums[kTreeWaves][kGroup][kD + 4];        // (rows padded: banks)
    struct {
      float m[kMostPairs], l[kMostPairs];
    } parts;
  };
  float back[C][kGroup], slope[C][kGroup];
  int draft[C][kGroup];
  uint64_t family[kMaxDrafts];                     // a draft and its ancestors
  int depth[kMaxDrafts];
  float m[kTreeWaves][kGroup], l[kTreeWaves][kGroup];
  float top[C * kGroup], total[C * kGroup];
  int scan[2][kTreeWaves], found[4];
  unsigned arrived;
};

// This thread's number plus those of the threads before it; `total`: of all.
template <int W>
__device__ inline int scan_all(int x, int* space, int& total) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int incl = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(incl, o, 64);
    incl += lane >= o ? up : 0;
  }
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

template <class M, int QT, int C>
__global__ __launch_bounds__(64 * kTreeWaves, 2) void tree_kernel(TreeArgs a) {
  constexpr int W = kTreeWaves, NT = 64 * W, TT = M::kTokens, NM = M::kMine;
  using Space = TreeSpace<M, QT, C>;
  using Query = typename Space::Query;
  constexpr int NF = Space::kPieces;
  constexpr bool kHasBack = sizeof(Query) != sizeof(Query::t);
  __shared__ Space sh;
  const PagedArgs& p = a.p;
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int heads = p.n_kv_heads;
  // The column blocks of one run read the same tokens: they are on one XCD (workgroups go to the
  // eight in turn) at one time, and meet in its L2.
  const int block = (int)blockIdx.x;
  const int unit = (block >> 3) / a.blocks * 8 + (block & 7), cb = (block >> 3) % a.blocks;
  const auto slots = __builtin_amdgcn_make_buffer_rsrc(p.parts, (short)0, p.parts_bytes, kRsrcWord3);

  auto cached = [&](int b) { return min(max(p.seq_len[b], 0), p.len_max); };
  auto drafted = [&](int b) {
    return a.n_draft ? min(max(a.n_draft[b], 0), a.drafts) : a.drafts;
  };
  auto tiles_of = [&](int b) {
    const int m = drafted(b);
    return row_tiles(cached(b) + m, window_of(p.window, m), p.sink, TT);
  };

  // The runs: every row (a sequence and KV head, all columns) in runs of at most `most` tiles.
  const int each = (p.batch + NT - 1) / NT;
  const int b0 = min(tid * each, p.batch), b1 = min(b0 + each, p.batch);
  int seq = 0, runs_before = 0, shared_before = 0, most;
  RowTiles rt;
  const int cap_parts = kMostPairs / a.block_cols;
  if (p.batch == 1) {
    if (drafted(0) == 0) return;                   // (uniform)
    rt = tiles_of(0);
    most = W * smallest_rounds(rt.n * heads, rt.n, heads, a.units, W,
                               [&](int q) { return heads * runs_of(rt.n, q); });
    most = max(most, runs_of(rt.n, cap_parts));
  } else {
    int mine = 0, longest = 0, rows = 0, tiles;
    for (int b = b0; b < b1; ++b) {
      const int t = drafted(b) ? tiles_of(b).n : 0;
      mine += t;
      rows += t > 0;
      longest = max(longest, t);
    }
    scan_all<W>(mine, sh.scan[0], tiles);
    scan_all<W>(rows, sh.scan[1], rows);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) longest = max(longest, __shfl_xor(longest, o, 64));
    __syncthreads();
    if (lane == 0) sh.scan[0][wave] = longest;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) longest = max(longest, sh.scan[0][w]);
    longest = __builtin_amdgcn_readfirstlane(longest);
    if (tiles == 0) return;                        // (uniform)
    auto runs = [&](int q) {
      int r = 0, all;
      for (int b = b0; b < b1; ++b) r += drafted(b) ? runs_of(tiles_of(b).n, q) : 0;
      scan_all<W>(r, sh.scan[0], all);
      return heads * all;
    };
    if (rows * heads <= a.units)
      most = W * smallest_rounds(tiles * heads, longest, rows * heads, a.units, W, runs);
    else
      most = max((int)(((int64_t)tiles * heads + a.units - 1) / a.units), kRoundsMin * W);
    most = max(most, runs_of(longest, cap_parts));
    // Which sequence has this run, and the runs and the shared rows' runs before it.
    int r = 0, s = 0, total;
    for (int b = b0; b < b1; ++b) {
      const int k = drafted(b) ? runs_of(tiles_of(b).n, most) : 0;
      r += heads * k;
      s += k > 1 ? heads * k : 0;
    }
    const int incl = scan_all<W>(r, sh.scan[0], total);
    int spare, at_shared = scan_all<W>(s, sh.scan[1], spare) - s;
    if (unit >= total) return;                     // (uniform)
    int at = incl - r;
    if (unit >= at && unit < incl) {               // (one thread)
      int b = b0;
      for (;; ++b) {
        const int k = drafted(b) ? runs_of(tiles_of(b).n, most) : 0;
        if (unit < at + heads * k) break;
        at += heads * k;
        at_shared += k > 1 ? heads * k : 0;
      }
      sh.found[0] = b;
      sh.found[1] = at;
      sh.found[2] = at_shared;
    }
    __syncthreads();
    seq = __builtin_amdgcn_readfirstlane(sh.found[0]);
    runs_before = __builtin_amdgcn_readfirstlane(sh.found[1]);
    shared_before = __builtin_amdgcn_readfirstlane(sh.found[2]);
    rt = tiles_of(seq);
  }
  const int parts = runs_of(rt.n, most);
  const int kvh = (unit - runs_before) % heads, part = (unit - runs_before) / heads;
  const int len = cached(seq), m = drafted(seq), G = p.G;
  const int columns = min(m * G - cb * a.block_cols, a.block_cols);
  if (part >= parts || columns <= 0) return;       // (uniform)
  const int groups = (columns + kGroup - 1) / kGroup;
  const int first = run_begin(rt.n, parts, part), last = run_begin(rt.n, parts, part + 1);
  const int end = len + m;
  const int lo = p.window > 0 ? max(0, end - window_of(p.window, m)) : 0;

  // Queries, and who descends from whom.
  Query own;
  auto column = [&](int c) { return cb * a.block_cols + c * kGroup + n; };
  auto fetch_query = [&](int c, Query& q) {
    const bool on = c * kGroup + n < columns;
    const int x = on ? column(c) : cb * a.block_cols, i = x / G, j = x - i * G;
    q.load(p.q, p.q_dtype,
           ((int64_t)seq * a.drafts + i) * p.q_stride + (int64_t)(kvh * G + j) * kD, on, g);
    if (g == 0) {
      sh.draft[c][n] = i;
      sh.slope[c][n] = p.slopes && on ? p.slopes[kvh * G + j] * kLog2e : 0.f;
    }
  };
  if constexpr (C == 1) {
    fetch_query(0, own);                           // (every wave its own registers)
  } else if (wave < groups) {
    fetch_query(wave, own);
    v4u piece[NF];
    __builtin_memcpy(piece, &own.t, sizeof own.t);
#pragma unroll
    for (int f = 0; f < NF; ++f) sh.q[wave][f][lane] = piece[f];
    if constexpr (kHasBack) {
      if (g == 0) sh.back[wave][n] = own.back;
    }
  }
  if (wave == W - 1) {
    int up = lane < m ? (a.parent ? a.parent[(int64_t)seq * a.drafts + lane] : lane - 1) : -1;
    up = up < lane ? max(up, -1) : -1;
    uint64_t family = (uint64_t)1 << lane;
#pragma unroll
    for (int d = 1; d < kMaxDrafts; d <<= 1) {     // ancestors up to 2 d - 1 steps away
      const int from = max(up, 0);
      const uint64_t theirs = __shfl(family, from, 64);
      const int higher = __shfl(up, from, 64);
      family |= up >= 0 ? theirs : 0;
      up = up >= 0 ? higher : -1;
    }
    sh.family[lane] = family;
    sh.depth[lane] = __popcll(family) - 1;
  }

  // Pages, keys and values.
  typename M::Keys key;
  typename M::Values val;
  const int32_t* row = p.table + seq * p.table_stride;
  auto page_of = [&](int t) {
    const int i = t >> p.page_shift;
    return i < p.max_pages ? row[i] : -1;
  };
  auto exists = [&](int page) { return (page >= 0) & (page < p.n_pages); };
  auto slot_of = [&](int t, int page) {
    return kvh * p.head_stride + (exists(page) ? page : 0) * p.page_stride +
           (t & ((1 << p.page_shift) - 1)) * p.tok_stride;
  };
  auto load_keys = [&](int t0, int page) {
    key.load(p.k + slot_of(t0 + M::key_token(0, n), page), p.tok_stride, g);
  };
  auto load_values = [&](int t0, int page) {
    val.load(p.v + slot_of(t0 + NM * g, page), p.tok_stride, n);
  };
  auto key_page = [&](int t0) { return page_of(t0 + 8 * M::key_block(n)); };
  auto value_page = [&](int t0) { return page_of(t0 + 8 * M::value_block(g)); };
  const int begin = first + wave;
  int t0 = rt.token(min(begin, last - 1), TT), t1 = rt.token(min(begin + W, last - 1), TT);
  int vp = value_page(t0), kp1 = key_page(t1), vp1 = value_page(t1);
  if (begin < last) {
    load_keys(t0, key_page(t0));
    load_values(t0, vp);
  }
  __syncthreads();

  v4f acc[C][8];
  float m_run[C], l_run[C], back[C];
  unsigned seen = 0u;                              // bit c: any token attended by the lane's column
#pragma unroll
  for (int c = 0; c < C; ++c) {
    m_run[c] = -INFINITY;
    l_run[c] = 0.f;
    back[c] = 1.f;
    if constexpr (C > 1 && kHasBack) back[c] = sh.back[c][n];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[c][j] = (v4f){0.f, 0.f, 0.f, 0.f};
  }
  for (int i = begin; i < last; i += W) {
    const bool more = i + W < last;
    float z[C][NM];
    // (the queries are read here each time: they have no room in registers)
    if constexpr (C > 1) asm volatile("" ::: "memory");
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (c >= groups) continue;                   // (uniform)
      if constexpr (C == 1) {
        M::template scores<QT>(key, own, z[c]);
      } else {
        Query q;
        v4u piece[NF];
#pragma unroll
        for (int f = 0; f < NF; ++f) piece[f] = sh.q[c][f][lane];
        __builtin_memcpy(&q.t, piece, sizeof q.t);
        if constexpr (kHasBack) q.back = back[c];
        M::template scores<QT>(key, q, z[c]);
      }
    }
    if (more) load_keys(t1, kp1);
    const int t2 = rt.token(min(i + 2 * W, last - 1), TT);
    const int kp2 = key_page(t2), vp2 = value_page(t2);
    // A tile that all columns attend as a whole needs no masks: the deepest draft stands at most
    // at end - 1.
    const bool there = exists(vp);
    const bool whole = t0 + TT <= len && (p.window == 0 || t0 > end - 1 - p.window || t0 + TT <= p.sink) &&
                       __builtin_amdgcn_ballot_w64(!there) == 0;
    unsigned dirty = 0u;                           // bit e: token NM g + e of the tile
    if (!whole) {
#pragma unroll
      for (int e = 0; e < NM; ++e) {
        val.keep(e, there & (t0 + NM * g + e < end) &
                        ((t0 + NM * g + e >= lo) | (t0 + NM * g + e < p.sink)));
        dirty |= M::bad(val, e) ? 1u << e : 0u;
      }
    }
    unsigned on_bits[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      on_bits[c] = ~0u;
      if (c >= groups) continue;                   // (uniform)
      if (p.cap > 0.f) {
        const float in = p.scale / p.cap, out = p.cap * kLog2e;
#pragma unroll
        for (int e = 0; e < NM; ++e) z[c][e] = out * tanh_of(z[c][e] * in);
      } else {
#pragma unroll
        for (int e = 0; e < NM; ++e) z[c][e] *= p.scale * kLog2e;
      }
      if (p.slopes || !whole) {
        const int draft = sh.draft[c][n], pos = len + sh.depth[draft];
        const uint64_t family = sh.family[draft];
        const float slope = sh.slope[c][n];
        if (!whole) on_bits[c] = 0u;
#pragma unroll
        for (int e = 0; e < NM; ++e) {
          const int t = t0 + NM * g + e;
          const int j = min(max(t - len, 0), kMaxDrafts - 1);
          const int at = whole || t < len ? t : len + sh.depth[j];
          if (p.slopes) z[c][e] -= slope * (float)(pos - at);
          if (!whole) {
            // (no short circuits: selects, not branches)
            const bool kin = (t < len) | ((t < end) & (bool)(family >> j & 1));
            const bool near = (p.window == 0) | (pos - at < p.window) | (t < p.sink);
            const bool on = there & kin & near;
            z[c][e] = on ? z[c][e] : -INFINITY;
            on_bits[c] |= on ? 1u << e : 0u;
          }
        }
      }
      seen |= on_bits[c] ? 1u << c : 0u;
      float top = z[c][0];
#pragma unroll
      for (int e = 1; e < NM; ++e) top = fmaxf(top, z[c][e]);
      top = over_groups_max(top) - kBelow<M>;
      if (__builtin_amdgcn_ballot_w64(top > m_run[c] + kSlack<M>)) {
        const float next = top > m_run[c] + kSlack<M> ? top : m_run[c];
        const float ref = next == -INFINITY ? 0.f : next;
        const float sa = __builtin_amdgcn_exp2f(m_run[c] - ref);    // (0 at the first tile)
        l_run[c] *= sa;
        m_run[c] = next;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[c][j] *= sa;
      }
      const float ref = m_run[c] == -INFINITY ? 0.f : m_run[c];
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < NM; ++e) {
        z[c][e] = __builtin_amdgcn_exp2f(z[c][e] - ref);
        sum += z[c][e];
      }
      l_run[c] += sum;
    }
    // Values that are not finite count for the columns that attend them and for no others (0 times
    // them is NaN): such tokens, if there are any, one by one, with a choice behind the product.
    if (__builtin_amdgcn_ballot_w64(dirty != 0u)) {
      for (int tok = 0; tok < TT; ++tok) {
        const int ge = tok / NM, te = tok % NM;
        if (!__builtin_amdgcn_ballot_w64(g == ge && (dirty >> te & 1u))) continue;
        typename M::Values one = val;              // the token's row, in place of the first
#pragma unroll
        for (int e = 1; e < NM; ++e) {
          M::take(one, val, e, e == te);
          one.keep(e, false);
        }
        one.keep(0, g == ge);
        typename M::Turned turned;
        M::turn(one, turned);
#pragma unroll
        for (int c = 0; c < C; ++c) {
          if (c >= groups) continue;               // (uniform)
          float w[NM];
#pragma unroll
          for (int e = 0; e < NM; ++e) w[e] = 0.f;
#pragma unroll
          for (int e = 0; e < NM; ++e) w[0] = e == te ? z[c][e] : w[0];
          const bool on = __shfl(on_bits[c], n + 16 * ge, 64) >> te & 1u;
          const auto terms = M::split(w);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const v4f sum = M::add(turned, j, terms, acc[c][j]);
#pragma unroll
            for (int x = 0; x < 4; ++x) acc[c][j][x] = on ? sum[x] : acc[c][j][x];
          }
        }
        // (its row is zeros from here on)
#pragma unroll
        for (int e = 0; e < NM; ++e) val.keep(e, !(g == ge && e == te));
      }
    }
    typename M::Turned turned;
    M::turn(val, turned);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (c >= groups) continue;                   // (uniform)
      const auto terms = M::split(z[c]);
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[c][j] = M::add(turned, j, terms, acc[c][j]);
    }
    if (more) load_values(t1, vp1);
    t0 = t1, vp = vp1;
    t1 = t2, kp1 = kp2, vp1 = vp2;
  }

  // The waves' sums meet in LDS, group by group.
  const int64_t out_row = (int64_t)seq * a.drafts * p.n_q_heads + kvh * G;
  auto finish = [&](int col, int c4, float top, float total, v4f o) {
    const int x = cb * a.block_cols + col, i = x / G, j = x - i * G;
    const int64_t head = out_row + (int64_t)i * p.n_q_heads + j;
    const bool lost = top == kLowest && total == total;     // attended scores were all -infinity
    if (lost) o = (v4f){NAN, NAN, NAN, NAN};
    const v4f zero = {0.f, 0.f, 0.f, 0.f};
    reinterpret_cast<v4f*>(p.out)[head * (kD / 4) + c4] = total == 0.f ? zero : o / total;
    if (p.lse && c4 == 0)
      p.lse[head] = total == 0.f || lost ? -INFINITY : (top + log2f(total)) * kLn2;
  };
  const int shared = shared_before + kvh;          // the row's first slot; part q's is heads q further
  auto part_at = [&](int q, int col) {
    return (((shared + q * heads) * a.blocks + cb) * a.block_cols + col) * (int)sizeof(Partial);
  };
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (c >= groups) continue;                     // (uniform)
    __syncthreads();                               // the queries, or the last group's sums, are read
    float l = over_groups_sum(l_run[c]);
    float top = m_run[c];
    unsigned any = seen >> c & 1u;
    any |= __shfl_xor(any, 16, 64);
    any |= __shfl_xor(any, 32, 64);
    if (any && top == -INFINITY && l == 0.f) {     // (NaN scores: the sum is NaN)
      top = kLowest;
      l = 1.f;
    }
    if (g == 0) {
      sh.m[wave][n] = top;
      sh.l[wave][n] = l;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) sh.sums[wave][n][M::channel(j, i, g)] = acc[c][j][i];
    __syncthreads();
    const int h = tid / (kD / 4), c4 = tid % (kD / 4), col = c * kGroup + h;
    static_assert(NT == kGroup * (kD / 4), "a thread for every four channels of a group");
    float mm = sh.m[0][h];
#pragma unroll
    for (int w = 1; w < W; ++w) mm = fmaxf(mm, sh.m[w][h]);
    float ll = 0.f;
    v4f o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = sh.m[w][h] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sh.m[w][h] - mm);
      ll += sh.l[w][h] == 0.f ? 0.f : f * sh.l[w][h];
      o += f * *reinterpret_cast<const v4f*>(&sh.sums[w][h][4 * c4]);
    }
    if (col < columns) {
      if (parts == 1) {
        finish(col, c4, mm, ll, o);
      } else {
        const int off = part_at(part, col);
        __builtin_amdgcn_raw_buffer_store_b128((v4i)o, slots, off + 16 + 16 * c4, 0, kCoherent);
        if (c4 == 0)
          __builtin_amdgcn_raw_buffer_store_b128((v4i)(v4f){mm, ll, 0.f, 0.f}, slots, off, 0,
                                                 kCoherent);
      }
    }
  }
  if (parts == 1) return;

  // The last of the row's workgroups joins them, in the order of the parts.
  unsigned* counter = p.counters + ((int64_t)shared * a.blocks + cb) * kTreeCounterStride;
  __builtin_amdgcn_s_waitcnt(0);                   // this thread's stores are done
  __syncthreads();
  if (tid == 0)
    sh.arrived = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (sh.arrived != (unsigned)parts - 1u) return;  // (uniform)
  auto slot = [&](int q, int col, int off) {
    return (v4f)__builtin_amdgcn_raw_buffer_load_b128(slots, part_at(q, col) + off, 0, kCoherent);
  };
  for (int x = tid; x < columns * parts; x += NT) {
    const v4f ml = slot(x / columns, x % columns, 0);
    sh.parts.m[x] = ml[0];
    sh.parts.l[x] = ml[1];
  }
  __syncthreads();
  for (int col = tid >> 3; col < columns; col += NT / 8) {        // eight threads a column
    float top = -INFINITY, total = 0.f;
    for (int q = tid & 7; q < parts; q += 8)
      if (sh.parts.l[q * columns + col] != 0.f) top = fmaxf(top, sh.parts.m[q * columns + col]);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    const float ref = top == -INFINITY ? 0.f : top;
    for (int q = tid & 7; q < parts; q += 8) {
      const float l = sh.parts.l[q * columns + col];
      const float w = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(sh.parts.m[q * columns + col] - ref);
      total += l == 0.f ? 0.f : w * l;             // (NaN stays)
      sh.parts.m[q * columns + col] = w;
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) total += __shfl_xor(total, o, 64);
    if ((tid & 7) == 0) {
      sh.top[col] = top;
      sh.total[col] = total;
    }
  }
  __syncthreads();
  constexpr int U = 8;                             // parts in flight
  for (int x = tid; x < columns * (kD / 4); x += NT) {
    const int col = x / (kD / 4), c4 = x % (kD / 4);
    v4f o = {0.f, 0.f, 0.f, 0.f};
    for (int q0 = 0; q0 < parts; q0 += U) {
      v4f v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = slot(min(q0 + u, parts - 1), col, 16 + 16 * c4);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float w = q0 + u < parts ? sh.parts.m[(q0 + u) * columns + col] : 0.f;
        if (w != 0.f) o += w * v[u];
      }
    }
    finish(col, c4, sh.top[col], sh.total[col], o);
  }
  if (tid == 0) *counter = 0u;                     // as the next call expects it
}

// A (sequence, KV head)'s columns in blocks of nearly as many groups each.
struct Blocks {
  int blocks, cols;
};
Blocks blocks_of(int drafts, int G) {
  const int groups = (drafts * G + kGroup - 1) / kGroup;
  const int blocks = (groups + kMostGroups - 1) / kMostGroups;
  return {blocks, (groups + blocks - 1) / blocks * kGroup};
}
int units_of(int blocks) { return std::max(1, kTreeGroups / blocks); }

size_t tree_parts_bytes(const Blocks& b) {
  return (size_t)kTreeSlots * b.cols * sizeof(Partial);
}

}  // namespace

size_t tree_workspace_bytes(int, int drafts, int n_q_heads, int n_kv_heads) {
  return kTreeCountersBytes + tree_parts_bytes(blocks_of(drafts, n_q_heads / n_kv_heads));
}

bool tree_fits(int64_t batch, int drafts, int n_q_heads, int n_kv_heads) {
  const int64_t columns = (int64_t)drafts * (n_q_heads / n_kv_heads);
  if (columns > kMaxColumns) return false;
  const Blocks b = blocks_of(drafts, n_q_heads / n_kv_heads);
  return (batch * n_kv_heads + kTreeGroups + 8) * b.blocks <= kMaxTreeGroups;
}

aatc_status launch_tree(TreeArgs a, aatc_dtype c_dtype, void* workspace, void* stream) {
  const Blocks b = blocks_of(a.drafts, a.p.G);
  a.blocks = b.blocks;
  a.block_cols = b.cols;
  a.units = units_of(b.blocks);
  a.p.counters = static_cast<unsigned*>(workspace);
  a.p.parts = reinterpret_cast<Partial*>(static_cast<char*>(workspace) + kTreeCountersBytes);
  a.p.parts_bytes = (int)tree_parts_bytes(b);
  // Rows that fit the chip are cut into runs that do; more rows into runs as long as the average
  // share: no more than `units` of them beyond one a row.
  const int rows = a.p.batch * a.p.n_kv_heads;
  const int64_t most = rows <= a.units ? a.units : (int64_t)rows + a.units;
  const int64_t grid = (most + 7) / 8 * 8 * b.blocks;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * kTreeWaves), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? AATC_OK : AATC_E_DEVICE;
  };
  auto launch_as = [&](auto m, auto qt) {
    using M = decltype(m);
    constexpr int QT = decltype(qt)::value;
    switch (b.cols / kGroup) {
      case 1: return launch(tree_kernel<M, QT, 1>);
      case 2: return launch(tree_kernel<M, QT, 2>);
      default: return launch(tree_kernel<M, QT, 4>);
    }
  };
  using One = std::integral_constant<int, 1>;
  using Three = std::integral_constant<int, 3>;
  const bool same = a.p.q_dtype == (int)c_dtype;
  auto launch_type = [&](auto far) {
    constexpr bool F = decltype(far)::value;
    switch (c_dtype) {
      case AATC_F32: return launch_as(Full32<F>{}, One{});
      case AATC_BF16:
        return same ? launch_as(Half16<__bf16, F>{}, One{}) : launch_as(Half16<__bf16, F>{}, Three{});
      default:
        return same ? launch_as(Half16<_Float16, F>{}, One{})
                    : launch_as(Half16<_Float16, F>{}, Three{});
    }
  };
  return launch_type(std::false_type{});
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
  const int64_t groups = (pieces + 255) / 256;
  constexpr int kMost = 65535;                     // sequences of a launch
  if (groups > (1 << 23)) return AATC_E_UNSUPPORTED;
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
