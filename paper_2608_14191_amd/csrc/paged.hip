// Attention of one new token per sequence over a paged cache at input precision.
//
// For query head j of sequence b, over the attended tokens t of its pages:
//   z_t = cap tanh(scale q . k_t / cap) - slope (len - 1 - t),   o = sum_t softmax(z)_t v_t.
//
// One pass with a running maximum and sum.  A wave takes a tile of 32 tokens (16 in float32) of
// one KV head against up to 16 query heads on the matrix cores, scores = K Q^T and then
// O^T += V^T P^T.  The tokens of the two 16-row blocks of a score tile are chosen so that the
// scores that a lane ends with (one head, tokens 8 g .. 8 g + 7) are the very ones it has to
// bring to the second product: nothing crosses lanes but the maximum.  K rows go from memory to
// the operand registers as they are; V rows are loaded as whole rows (a lane: 16 bytes of eight
// tokens) and turned 8 x 8 in the lane's own registers.
//
// Precision: products of the stored values with fp32 sums.  P is split into terms of the
// cache's type that add up to (nearly) its 24 bits: three in bf16, two in f16 (with the maximum
// taken 14 lower, so that small weights stay off f16's denormals); queries of another type than
// the cache's into three.
//
// A row is a sequence, a KV head and up to 16 of its query heads.  How the rows are shared out
// (paged_plan.h) follows from the lengths, which only the device knows.  A row that several
// workgroups or waves share is joined by the last of them to arrive, in the order of the parts.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "paged.h"
#include "paged_join.h"
#include "paged_plan.h"
#include "paged_tile.h"
#include "params.h"

namespace aatc {
namespace {

// Runs (few rows): eight waves a workgroup, one workgroup a compute unit, so that a row has few
// parts to join (1 x 32768 tokens, 8 KV heads, float16: 27.7 us, with four waves and twice as many
// 30.5; shorter rows would gain by those: 1 x 4000 bf16 13.0 and 10.7).
// Lines (many rows): four waves, two workgroups a compute unit, whose row changes cover each
// other (48 x 2052 tokens, 8 KV heads, float32: 142.2 us, with eight waves 156.3).
constexpr int kRunWaves = 8, kRunGroups = 256;
constexpr int kLineWaves = 4, kLineGroups = 512;
constexpr int kMaxRunRows = 256;                  // a workgroup each at least
// The workspace: arrival counters, one for each worker (a shared row's is its first worker's: no
// worker has more than one row that others go on with), in one place whatever the shape of a call,
// then part slots of slot_heads partials.  Counters are 256 bytes apart (their atomics would queue
// on one cache line) and left at zero.
constexpr int kWorkers = kLineGroups * kLineWaves, kCounterStride = 64;
constexpr size_t kCountersBytes = (size_t)kWorkers * kCounterStride * sizeof(unsigned);

// A row: query heads h0 .. h0 + heads - 1 of sequence `seq` on KV head `kvh`.
struct Row {
  int len, kvh, h0, heads;
  int64_t q_row;
};
__device__ inline Row row_of(const PagedArgs& a, int seq, int row) {
  Row r;
  r.len = min(max(a.seq_len[seq], 0), a.len_max);
  r.kvh = row / a.hg;
  r.h0 = r.kvh * a.G + (row % a.hg) * kPagedHeads;
  r.heads = min(kPagedHeads, (r.kvh + 1) * a.G - r.h0);
  r.q_row = (int64_t)seq * a.n_q_heads + r.h0;
  return r;
}

// A wave's way through its rows.  Where a workgroup has several, the pages of the next one's first
// tiles are fetched before a row is begun, and its queries, keys and values when that is done, under
// the row's join (192 rows of 63 tiles at most, as lines: 44.2 us, 46.4 without).
template <class M, int QT>
struct Walk {
  static constexpr int TT = M::kTokens, NM = M::kMine;
  // (Registers: 16-bit caches with queries of their own type have room for a row's first keys and
  // values under the last one's join.)
  static constexpr bool kEarly = QT == 1 && TT == 32;
  const PagedArgs& a;
  const int n = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
  typename M::template Query<QT> q;
  typename M::Keys key;
  typename M::Values val;
  float slope;

  // The tiles first, first + step .. below last of a row.
  struct Share {
    Row r;
    RowTiles rt;
    int seq, first, last, step;
    int t0, t1;                                    // its first two tiles' tokens and their pages
    int kp, vp, kp1, vp1;                          // (keys' and values' blocks of the lane)
  };

  __device__ explicit Walk(const PagedArgs& args) : a(args) {}

  // Page of the 8-token block `blk` of the tile at token t0 (-1: none there).
  __device__ int page_of(int seq, int t0, int blk) const {
    const int i = (t0 + 8 * blk) >> a.page_shift;
    return i < a.max_pages ? a.table[seq * a.table_stride + i] : -1;
  }
  __device__ bool exists(int page) const { return (page >= 0) & (page < a.n_pages); }
  __device__ int64_t slot_of(int t, int page) const {
    return (exists(page) ? page : 0) * a.page_stride + (t & ((1 << a.page_shift) - 1)) * a.tok_stride;
  }
  __device__ void load_keys(const Share& s, int t0, int page) {
    key.load(a.k + s.r.kvh * a.head_stride + slot_of(t0 + M::key_token(0, n), page), a.tok_stride, g);
  }
  __device__ void load_values(const Share& s, int t0, int page) {
    val.load(a.v + s.r.kvh * a.head_stride + slot_of(t0 + NM * g, page), a.tok_stride, n);
  }

  __device__ Share share(int seq, int row, const RowTiles& rt, int first, int last, int step) const {
    Share s;
    s.r = row_of(a, seq, row);
    s.rt = rt;
    s.seq = seq;
    s.first = first;
    s.last = last;
    s.step = step;
    s.t0 = rt.token(min(first, last - 1), TT);
    s.t1 = rt.token(min(first + step, last - 1), TT);
    s.kp = page_of(seq, s.t0, M::key_block(n));
    s.vp = page_of(seq, s.t0, M::value_block(g));
    s.kp1 = page_of(seq, s.t1, M::key_block(n));
    s.vp1 = page_of(seq, s.t1, M::value_block(g));
    return s;
  }

  __device__ void fetch(const Share& s) {
    const bool on = n < s.r.heads;
    q.load(a.q, a.q_dtype,
           (int64_t)s.seq * a.q_stride + (int64_t)(s.r.h0 + min(n, s.r.heads - 1)) * kD, on, g);
    slope = a.slopes && on ? a.slopes[s.r.h0 + n] * kLog2e : 0.f;
    if (s.first < s.last) {
      load_keys(s, s.t0, s.kp);
      load_values(s, s.t0, s.vp);
    }
  }

  __device__ void run(const Share& s, RowPart& out) {
    const int len = s.r.len, lo = a.window > 0 ? max(0, len - a.window) : 0;
    const int last = s.last, step = s.step;
    int t0 = s.t0, vp = s.vp, t1 = s.t1, kp1 = s.kp1, vp1 = s.vp1;
    float m_run = -INFINITY, l_run = 0.f;
    bool seen = false;                             // any token attended (of the wave's, uniform)
    v4f(&acc)[8] = out.acc;
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = (v4f){0.f, 0.f, 0.f, 0.f};
    for (int i = s.first; i < last; i += step) {
      // Two tiles ahead: pages; one tile ahead: keys and values.
      const bool more = i + step < last;
      float z[NM];
      M::template scores<QT>(key, q, z);
      if (more) load_keys(s, t1, kp1);
      const int t2 = s.rt.token(min(i + 2 * step, last - 1), TT);
      const int kp2 = page_of(s.seq, t2, M::key_block(n)), vp2 = page_of(s.seq, t2, M::value_block(g));
      if (a.cap > 0.f) {
        const float in = a.scale / a.cap, back = a.cap * kLog2e;
#pragma unroll
        for (int e = 0; e < NM; ++e) z[e] = back * tanh_of(z[e] * in);
      } else {
#pragma unroll
        for (int e = 0; e < NM; ++e) z[e] *= a.scale * kLog2e;
      }
      if (a.slopes) {
#pragma unroll
        for (int e = 0; e < NM; ++e) z[e] -= slope * (float)(len - 1 - (t0 + NM * g + e));
      }
      // A tile that is attended as a whole needs no masks.
      const bool there = exists(vp);
      const bool whole = t0 + TT <= len && (t0 >= lo || t0 + TT <= a.sink) &&
                         __builtin_amdgcn_ballot_w64(!there) == 0;
      if (!whole) {
        bool any = false;
#pragma unroll
        for (int e = 0; e < NM; ++e) {
          const int t = t0 + NM * g + e;
          // (no short circuits: selects, not branches)
          const bool on = there & (t < len) & ((t >= lo) | (t < a.sink));
          z[e] = on ? z[e] : -INFINITY;
          val.keep(e, on);
          any |= on;
        }
        seen |= __builtin_amdgcn_ballot_w64(any) != 0;
      } else {
        seen = true;
      }
      float m = z[0];
#pragma unroll
      for (int e = 1; e < NM; ++e) m = fmaxf(m, z[e]);
      m = fmaxf(m_run, reference_of<M>(over_groups_max(m)));
      const float ref = m == -INFINITY ? 0.f : m;
      const float sa = __builtin_amdgcn_exp2f(m_run - ref);    // (0 at the first tile)
      float p[NM], sum = 0.f;
#pragma unroll
      for (int e = 0; e < NM; ++e) {
        p[e] = __builtin_amdgcn_exp2f(z[e] - ref);
        sum += p[e];
      }
      l_run = l_run * sa + sum;
      m_run = m;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] *= sa;
      M::accumulate(val, p, acc);
      if (more) load_values(s, t1, vp1);
      t0 = t1, vp = vp1;
      t1 = t2, kp1 = kp2, vp1 = vp2;
    }
    out.m = m_run;
    out.l = over_groups_sum(l_run);
    if (seen && out.m == -INFINITY && out.l == 0.f) {     // (NaN scores: the sum is NaN)
      out.m = kLowest;
      out.l = 1.f;
    }
  }
};

// Lines of waves: every wave takes its tiles, or its row, for itself.  Rows that a wave has whole
// need no join; the others are joined by the last of their waves.  `before`, `mine`: tiles before
// and of this thread's sequences b0 ...
template <class M, int QT>
__device__ __forceinline__ void line_of_waves(const PagedArgs& a, LineWay way, int total,
                                              int before, int mine, int b0, int (*found)[2],
                                              __amdgpu_buffer_rsrc_t slots) {
  constexpr int W = kLineWaves;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int me = (int)blockIdx.x * W + wave;
  const int rows = a.n_kv_heads * a.hg, quota = way.quota;
  auto tiles_of = [&](int b) {
    return row_tiles(min(max(a.seq_len[b], 0), a.len_max), a.window, a.sink, M::kTokens);
  };
  int seq, row, start, end;
  RowTiles rt;
  if (way.whole) {
    if (me >= a.batch * rows) return;
    seq = me / rows;
    row = me % rows;
    rt = tiles_of(seq);
    start = me * quota;
    end = start + rt.n;
  } else {
    for (int w = 0; w < W; ++w) {                  // (one thread finds each: no other has the tile)
      const int x = ((int)blockIdx.x * W + w) * quota;
      if (x >= before && x < before + mine) {
        int b = b0, at = before;
        for (;; ++b) {
          const int t = tiles_of(b).n * rows;
          if (x < at + t) break;
          at += t;
        }
        found[w][0] = b;
        found[w][1] = at;
      }
    }
    __syncthreads();
    const int begin = me * quota;
    if (begin >= total) return;
    end = min(begin + quota, total);
    seq = __builtin_amdgcn_readfirstlane(found[wave][0]);
    const int at = __builtin_amdgcn_readfirstlane(found[wave][1]);
    rt = tiles_of(seq);
    row = (begin - at) / rt.n;
    start = at + row * rt.n;
  }
  Walk<M, QT> walk(a);
  for (;;) {
    const auto now = walk.share(seq, row, rt, max(me * quota - start, 0), min(end - start, rt.n), 1);
    const Row& r = now.r;
    const RowShare share = row_share(start, rt.n, quota);
    const int parts = share.last - share.first + 1;
    RowPart x;
    walk.fetch(now);
    walk.run(now, x);
    auto part_at = [&](int p, int h) {
      return (part_slot(share.first + p, start, quota) * a.slot_heads + h) * (int)sizeof(Partial);
    };
    if (n < r.heads) {
#pragma unroll
      for (int j = 0; j < 8; j += 4)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c = M::channel(j, i, g);
          const v4f o = {x.acc[j][i], x.acc[j + 1][i], x.acc[j + 2][i], x.acc[j + 3][i]};
          if (parts == 1)
            finish_row(a, r.q_row + n, c / 4, x.m, x.l, o);
          else
            __builtin_amdgcn_raw_buffer_store_b128((v4i)o, slots,
                                                   part_at(me - share.first, n) + 16 + 4 * c, 0,
                                                   kCoherent);
        }
      if (parts > 1 && g == 0)
        __builtin_amdgcn_raw_buffer_store_b128((v4i)(v4f){x.m, x.l, 0.f, 0.f}, slots,
                                               part_at(me - share.first, n), 0, kCoherent);
    }
    if (parts > 1) {
      unsigned* counter = a.counters + share.first * kCounterStride;
      __builtin_amdgcn_s_waitcnt(0);               // the wave's stores are done
      unsigned before_me = 0u;
      if (lane == 0)
        before_me = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (__builtin_amdgcn_readfirstlane(before_me) == (unsigned)parts - 1u) {
        constexpr int U = 4;                       // parts in flight
        for (int u = lane; u < r.heads * (kD / 4); u += 64) {
          const int h = u / (kD / 4), c4 = u % (kD / 4);
          float m = -INFINITY, l = 0.f;
          v4f o = {0.f, 0.f, 0.f, 0.f};
          for (int p0 = 0; p0 < parts; p0 += U) {
            v4f ml[U], po[U];
#pragma unroll
            for (int p = 0; p < U; ++p) {
              const int at = part_at(min(p0 + p, parts - 1), h);
              ml[p] = (v4f)__builtin_amdgcn_raw_buffer_load_b128(slots, at, 0, kCoherent);
              po[p] = (v4f)__builtin_amdgcn_raw_buffer_load_b128(slots, at + 16 + 16 * c4, 0, kCoherent);
            }
#pragma unroll
            for (int p = 0; p < U; ++p) {
              const bool on = (p0 + p < parts) & (ml[p][1] != 0.f);    // (NaN counts)
              const float top = on ? fmaxf(m, ml[p][0]) : m;
              const float ref = top == -INFINITY ? 0.f : top;
              const float fa = __builtin_amdgcn_exp2f(m - ref);
              const float fb = on ? __builtin_amdgcn_exp2f(ml[p][0] - ref) : 0.f;
              l = l * fa + (on ? ml[p][1] * fb : 0.f);
              o = o * fa + fb * po[p];
              m = top;
            }
          }
          finish_row(a, r.q_row + h, c4, m, l, o);
        }
        if (lane == 0) *counter = 0u;              // as the next call expects it
      }
    }
    start += rt.n;
    if (start >= end) return;
    if (++row == rows) {
      row = 0;
      ++seq;
      rt = tiles_of(seq);
    }
  }
}

template <class M, int QT, bool RUNS>
__global__ __launch_bounds__(64 * (RUNS ? kRunWaves : kLineWaves), 2) void paged_kernel(PagedArgs a) {
  constexpr int W = RUNS ? kRunWaves : kLineWaves, NT = 64 * W;
  constexpr int TT = M::kTokens, NM = M::kMine;
  __shared__ JoinSpace<W, RUNS ? kRunGroups : kLineGroups> sh;
  __shared__ int scan[2][W], found[W][2];
  __shared__ unsigned arrived;
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int block = (int)blockIdx.x, grid = (int)gridDim.x;
  const int rows = a.n_kv_heads * a.hg;            // of a sequence
  // Part slots, Partial [slot_heads] each, stored and loaded where every compute unit sees them.
  const auto slots = __builtin_amdgcn_make_buffer_rsrc(a.parts, (short)0, a.parts_bytes, kRsrcWord3);

  auto length = [&](int b) { return min(max(a.seq_len[b], 0), a.len_max); };
  auto tiles_of = [&](int b) { return row_tiles(length(b), a.window, a.sink, TT); };

  // This workgroup's share: tiles first .. last - 1 of row `row` of sequence `seq`, part `part` of
  // `parts`.  Lines: the row begins at tile `start` of the line, the share ends at `end`.
  int seq = 0, row = 0, first, last, part = 0, parts = 1;
  int quota = 0, start = 0, end = 0;
  RowTiles rt;
  if constexpr (RUNS) {
    const int all = a.batch * rows;
    if (a.batch == 1) {
      rt = tiles_of(0);
      parts = runs_of(rt.n, W * smallest_rounds(rt.n * rows, rt.n, rows, grid, W, [&](int q) {
                        return rows * runs_of(rt.n, q);
                      }));
      row = block / parts;
      part = block % parts;
      if (row >= rows) return;                     // (uniform)
    } else {
      // Some sequences a lane; every wave does the same.
      constexpr int S = kMaxRunRows / 64;
      int n_of[S], longest = 0, tiles = 0;
#pragma unroll
      for (int i = 0; i < S; ++i) {
        n_of[i] = lane + 64 * i < a.batch ? tiles_of(lane + 64 * i).n : 0;
        longest = max(longest, n_of[i]);
        tiles += n_of[i];
      }
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        tiles += __shfl_xor(tiles, o, 64);
        longest = max(longest, __shfl_xor(longest, o, 64));
      }
      longest = __builtin_amdgcn_readfirstlane(longest);
      tiles = __builtin_amdgcn_readfirstlane(tiles);
      const int q = W * smallest_rounds(tiles * rows, longest, all, grid, W, [&](int x) {
                      int v = 0;
#pragma unroll
                      for (int i = 0; i < S; ++i) v += runs_of(n_of[i], x);
#pragma unroll
                      for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
                      return rows * __builtin_amdgcn_readfirstlane(v);
                    });
      // Runs before each sequence; the one that has this workgroup's, and its first.
      int carry = 0, before = 0;
      seq = 0;
#pragma unroll
      for (int i = 0; i < S; ++i) {
        const int mine = rows * runs_of(n_of[i], q);
        int incl = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const int up = __shfl_up(incl, o, 64);
          incl += lane >= o ? up : 0;
        }
        incl += carry;
        carry = __builtin_amdgcn_readlane(incl, 63);
        const uint64_t past = __builtin_amdgcn_ballot_w64(incl <= block);
        seq += __popcll(past);
        if (past != ~(uint64_t)0 && carry > block && seq < 64 * (i + 1) && seq >= 64 * i)
          before = __builtin_amdgcn_readlane(incl - mine, seq - 64 * i);
      }
      if (block >= carry) return;                  // (uniform)
      rt = tiles_of(seq);
      parts = runs_of(rt.n, q);
      row = (block - before) / parts;
      part = (block - before) % parts;
    }
    first = run_begin(rt.n, parts, part);
    last = run_begin(rt.n, parts, part + 1);
  } else {
    // Every thread adds up a run of sequences, a scan over the workgroup.
    const int each = (a.batch + NT - 1) / NT;
    const int b0 = min(tid * each, a.batch), b1 = min(b0 + each, a.batch);
    int mine = 0, longest = 0;
    for (int b = b0; b < b1; ++b) {
      const int t = tiles_of(b).n;
      mine += t * rows;
      longest = max(longest, t);
    }
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(incl, o, 64);
      incl += lane >= o ? up : 0;
      longest = max(longest, __shfl_xor(longest, o, 64));
    }
    if (lane == 63) {
      scan[0][wave] = incl;
      scan[1][wave] = longest;
    }
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      incl += w < wave ? scan[0][w] : 0;
      total += scan[0][w];
      longest = max(longest, scan[1][w]);
    }
    total = __builtin_amdgcn_readfirstlane(total);
    longest = __builtin_amdgcn_readfirstlane(longest);
    const LineWay way = line_way(total, longest, a.batch * rows, grid, W);
    quota = way.quota;
    if (way.waves) {
      line_of_waves<M, QT>(a, way, total, incl - mine, mine, b0, found, slots);
      return;
    }
    if (way.whole) {
      if (block >= a.batch * rows) return;         // (uniform)
      seq = block / rows;
      row = block % rows;
      rt = tiles_of(seq);
      start = block * quota;
      end = start + rt.n;
      first = 0;
      last = rt.n;
    } else {
      const int begin = block * quota;
      if (begin >= total) return;                  // (uniform)
      end = min(begin + quota, total);
      int at = incl - mine;
      if (begin >= at && begin < incl) {           // (one thread: runs without tiles are empty)
        int b = b0;
        for (;; ++b) {
          const int t = tiles_of(b).n * rows;
          if (begin < at + t) break;
          at += t;
        }
        found[0][0] = b;
        found[0][1] = at;
      }
      __syncthreads();
      seq = __builtin_amdgcn_readfirstlane(found[0][0]);
      const int before = __builtin_amdgcn_readfirstlane(found[0][1]);
      rt = tiles_of(seq);
      row = (begin - before) / rt.n;
      start = before + row * rt.n;
      first = begin - start;
      last = min(end, start + rt.n) - start;
      const RowShare share = row_share(start, rt.n, quota);
      parts = share.last - share.first + 1;
      part = block - share.first;
    }
  }

  Walk<M, QT> walk(a);
  auto now = walk.share(seq, row, rt, first + wave, last, W);
  walk.fetch(now);
  for (;;) {
    const Row r = now.r;
    const int heads = r.heads;
    // The next row (lines).
    const int next_start = start + rt.n;
    const bool more = !RUNS && next_start < end;
    const bool turn = row + 1 == rows;
    const int next_seq = turn ? seq + 1 : seq, next_row = turn ? 0 : row + 1;
    auto next = now;
    if (more) {
      if (turn) rt = tiles_of(next_seq);
      next = walk.share(next_seq, next_row, rt, wave, min(end - next_start, rt.n), W);
    }
    RowPart mine;
    walk.run(now, mine);
    if (walk.kEarly && more) walk.fetch(next);

    // The waves' parts meet in LDS.
    if (g == 0) {
      sh.m[wave][n] = mine.m;
      sh.l[wave][n] = mine.l;
    }
    if (n < heads) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) sh.sums[wave][n][M::channel(j, i, g)] = mine.acc[j][i];
    }
    __syncthreads();

    auto finish = [&](int h, int c4, float m, float l, v4f o) {
      finish_row(a, r.q_row + h, c4, m, l, o);
    };
    auto part_at = [&](int p, int h) {
      const int w = block - part + p;
      const int slot = RUNS ? w : part_slot(w, start, quota);
      return (slot * a.slot_heads + h) * (int)sizeof(Partial);
    };
    for (int x = tid; x < heads * (kD / 4); x += NT) {
      const int h = x / (kD / 4), c4 = x % (kD / 4);
      float m = sh.m[0][h];
#pragma unroll
      for (int w = 1; w < W; ++w) m = fmaxf(m, sh.m[w][h]);
      float l = 0.f;
      v4f o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float f = sh.m[w][h] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sh.m[w][h] - m);
        l += sh.l[w][h] == 0.f ? 0.f : f * sh.l[w][h];
        o += f * *reinterpret_cast<const v4f*>(&sh.sums[w][h][4 * c4]);
      }
      if (parts == 1) {
        finish(h, c4, m, l, o);
      } else {
        const int off = part_at(part, h);
        __builtin_amdgcn_raw_buffer_store_b128((v4i)o, slots, off + 16 + 16 * c4, 0, kCoherent);
        if (c4 == 0)
          __builtin_amdgcn_raw_buffer_store_b128((v4i)(v4f){m, l, 0.f, 0.f}, slots, off, 0,
                                                 kCoherent);
      }
    }
    if (parts > 1) {
      unsigned* counter = a.counters + (block - part) * kCounterStride;
      __builtin_amdgcn_s_waitcnt(0);               // this thread's stores are done
      __syncthreads();
      if (tid == 0)
        arrived = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __syncthreads();
      if (arrived == (unsigned)parts - 1u) {
        join_parts(sh, parts, heads, finish, [&](int p, int h, int off) {
          return (v4f)__builtin_amdgcn_raw_buffer_load_b128(slots, part_at(p, h) + off, 0,
                                                            kCoherent);
        });
        if (tid == 0) *counter = 0u;               // as the next call expects it
      }
    }
    if (!more) return;
    __syncthreads();                               // LDS is read: the next row's parts go there
    if (!walk.kEarly) walk.fetch(next);
    start = next_start;
    seq = next_seq;
    row = next_row;
    now = next;
    const RowShare share = row_share(start, rt.n, quota);
    parts = share.last - share.first + 1;
    part = block - share.first;
  }
}

// Part slots of a call of `rows` rows: a workgroup of the runs has one, a worker of the lines two.
size_t parts_bytes(int64_t rows, int slot_heads) {
  const int slots = rows <= kRunGroups / 2 ? kRunGroups : 2 * kWorkers;
  return (size_t)slots * slot_heads * sizeof(Partial);
}

}  // namespace

size_t paged_workspace_bytes(int batch, int n_q_heads, int n_kv_heads) {
  const int G = n_q_heads / n_kv_heads, hg = (G + kPagedHeads - 1) / kPagedHeads;
  return kCountersBytes + parts_bytes((int64_t)batch * n_kv_heads * hg, std::min(G, kPagedHeads));
}

aatc_status launch_paged(PagedArgs a, aatc_dtype c_dtype, void* workspace, void* stream) {
  a.counters = static_cast<unsigned*>(workspace);
  a.parts = reinterpret_cast<Partial*>(static_cast<char*>(workspace) + kCountersBytes);
  const int tt = c_dtype == AATC_F32 ? Full32<false>::kTokens : Half16<__bf16, false>::kTokens;
  const int64_t rows = (int64_t)a.batch * a.n_kv_heads * a.hg;
  const int64_t most = rows * std::max(1, (a.len_max + tt - 1) / tt);
  // Runs for up to half the grid's rows, or up to all of it where no row can be long, by the width of
  // the table (one run a row then lasts as long as the longest: 256 rows up to 2000 tokens 41.4 us,
  // as lines 52.0; 240 rows up to 12000 tokens 201, as lines 161).
  const bool runs = rows <= kRunGroups / 2 || (rows <= kMaxRunRows && a.len_max <= 128 * tt);
  a.slot_heads = std::min(a.G, kPagedHeads);
  a.parts_bytes = (int)parts_bytes(rows, a.slot_heads);
  const int grid = (int)std::min<int64_t>(runs ? kRunGroups : kLineGroups, most);
  const hipStream_t st = (hipStream_t)stream;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * (runs ? kRunWaves : kLineWaves)), 0,
                       st, a);
    return hipGetLastError() == hipSuccess ? AATC_OK : AATC_E_DEVICE;
  };
  auto launch_as = [&](auto m, auto qt) {
    using M = decltype(m);
    constexpr int QT = decltype(qt)::value;
    return runs ? launch(paged_kernel<M, QT, true>) : launch(paged_kernel<M, QT, false>);
  };
  using One = std::integral_constant<int, 1>;
  using Three = std::integral_constant<int, 3>;
  const bool same = a.q_dtype == (int)c_dtype;
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
  return pools_far(a, c_dtype) ? launch_type(std::true_type{}) : launch_type(std::false_type{});
}

}  // namespace aatc
