// Sparse attention over a paged cache: the pages' bounds, the pages that a query can score highest
// in, and attention over those.
//
// A page's bound on a score sum_c q_c k_c is sum_c max(q_c hi_c, q_c lo_c), hi and lo the largest and
// smallest value of channel c in the page: with the positive and the negative part of q a product of
// 256 numbers, [q+ q-] . [hi lo].  All of them are held in 8 bits with powers of two as steps, so the
// product on the int8 matrix cores, the steps and the comparison are exact: the pages picked depend on
// no order of summation.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "paged_join.h"
#include "paged_plan.h"
#include "paged_tile.h"
#include "params.h"
#include "sparse.h"
#include "wave_scan.h"

namespace aatc {
namespace {

constexpr int kLowestStep = -50, kHighestStep = 100;

// The exponent of the smallest power of two, from 2^-50 on, of which 127 reach `top` (finite, >= 0).
__device__ inline int step_of(float top) {
  const uint32_t bits = __float_as_uint(top);
  const int e = (int)(bits >> 23) - 126 - ((bits & 0x7fffffu) <= 0x7e0000u ? 7 : 6);
  return max(e, kLowestStep);
}
__device__ inline float power_of_two(int e) {     // -126 <= e <= 127
  return __uint_as_float((uint32_t)(e + 127) << 23);
}

// --- bounds ---------------------------------------------------------------------------------------

// A wave takes a run of (page, KV head) pairs, one at a time: a row of 16 (32 in float32) lanes has a
// token, a lane 16 bytes of it; what the rows have meets in row swaps.  Reads every key once, past the
// caches: the memory bounds it (65536 tokens x 8 float32 heads: 5.9 TB/s), small pages the vector units.
// 16-bit values are compared as whole numbers in their order, two at a time.
constexpr int kBoundWaves = 4, kBoundGroups = 2048;

// Largest and smallest of what a lane has seen, channel by channel.
template <class T>
struct Extremes {                                  // 16 bits: eight channels, in pairs
  typedef int16_t v2 __attribute__((ext_vector_type(2)));
  static constexpr int N = 8;
  // The number that is larger the larger the value is (its own inverse); infinities and NaN lie at
  // either end.
  static constexpr int kInfinite = __is_same(T, _Float16) ? 0x7c00 : 0x7f80;
  v2 top[4], low[4];
  __device__ void clear() {
#pragma unroll
    for (int d = 0; d < 4; ++d) top[d] = (v2){-32768, -32768}, low[d] = (v2){32767, 32767};
  }
  static __device__ v2 pair(uint32_t x) { return __builtin_bit_cast(v2, x); }
  static __device__ uint32_t word(v2 x) { return __builtin_bit_cast(uint32_t, x); }
  __device__ void add(v4u x) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      v2 v = pair(x[d]);
      v ^= (v >> 15) & (v2){0x7fff, 0x7fff};
      top[d] = __builtin_elementwise_max(top[d], v);
      low[d] = __builtin_elementwise_min(low[d], v);
    }
  }
  __device__ void join_rows() {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      auto r = __builtin_amdgcn_permlane16_swap(word(top[d]), word(top[d]), false, false);
      top[d] = __builtin_elementwise_max(pair(r[0]), pair(r[1]));
      r = __builtin_amdgcn_permlane32_swap(word(top[d]), word(top[d]), false, false);
      top[d] = __builtin_elementwise_max(pair(r[0]), pair(r[1]));
      r = __builtin_amdgcn_permlane16_swap(word(low[d]), word(low[d]), false, false);
      low[d] = __builtin_elementwise_min(pair(r[0]), pair(r[1]));
      r = __builtin_amdgcn_permlane32_swap(word(low[d]), word(low[d]), false, false);
      low[d] = __builtin_elementwise_min(pair(r[0]), pair(r[1]));
    }
  }
  static __device__ float value(int16_t x) {
    const uint16_t bits = (uint16_t)(x ^ ((x >> 15) & 0x7fff));
    return (float)__builtin_bit_cast(T, bits);
  }
  __device__ float largest(int i) const { return value(top[i / 2][i % 2]); }
  __device__ float smallest(int i) const { return value(low[i / 2][i % 2]); }
  __device__ bool bad() const {
    bool b = false;
#pragma unroll
    for (int i = 0; i < N; ++i) b |= (top[i / 2][i % 2] >= kInfinite) | (low[i / 2][i % 2] <= ~kInfinite);
    return b;
  }
};
template <>
struct Extremes<float> {
  static constexpr int N = 4;
  float top[4], low[4];
  bool odd;
  __device__ void clear() {
    odd = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) top[i] = -INFINITY, low[i] = INFINITY;
  }
  __device__ void add(v4u x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float v = __uint_as_float(x[i]);
      odd |= !(fabsf(v) < INFINITY);
      top[i] = fmaxf(top[i], v);
      low[i] = fminf(low[i], v);
    }
  }
  __device__ void join_rows() {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(top[i]), __float_as_uint(top[i]), false, false);
      top[i] = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
      r = __builtin_amdgcn_permlane32_swap(__float_as_uint(low[i]), __float_as_uint(low[i]), false, false);
      low[i] = fminf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
  }
  __device__ float largest(int i) const { return top[i]; }
  __device__ float smallest(int i) const { return low[i]; }
  __device__ bool bad() const { return odd; }
};

template <class T>
__global__ __launch_bounds__(64 * kBoundWaves) void bounds_kernel(BoundsArgs a) {
  constexpr int W = kBoundWaves, NT = 64 * W;
  constexpr int N = Extremes<T>::N, L = kD / N;    // channels of a lane, lanes of a token
  constexpr int U = 16 / (64 / L);                 // loads of 16 tokens
  __shared__ int before[NT], sums[W];              // pages of the threads' rows up to their last
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int each = (a.rows + NT - 1) / NT;
  auto tokens = [&](const int32_t* x, int b) { return x ? min(max(x[b], 0), a.len_max) : 0; };
  // Pages that row b's new tokens fall into: `first` on, so many.
  auto pages_of = [&](int b, int& first) {
    const int from = tokens(a.held, b), to = tokens(a.wanted, b);
    first = from >> a.page_shift;
    return to > from ? ((to - 1) >> a.page_shift) + 1 - first : 0;
  };
  int mine = 0, skip;
  for (int b = min(tid * each, a.rows); b < min((tid + 1) * each, a.rows); ++b) mine += pages_of(b, skip);
  int incl = wave_scan_sum(mine);                  // (pages of all rows: below 2^30)
  if (lane == 63) sums[wave] = incl;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    incl += w < wave ? sums[w] : 0;
    total += sums[w];
  }
  before[tid] = incl;
  __syncthreads();
  // This wave's run of pairs, the heads of a page one after another.
  const int64_t items = (int64_t)__builtin_amdgcn_readfirstlane(total) * a.n_kv_heads;
  const int64_t waves = (int64_t)gridDim.x * W, me = (int64_t)blockIdx.x * W + wave;
  const int begin = (int)(items * me / waves), end = (int)(items * (me + 1) / waves);
  if (begin >= end) return;
  int at = begin / a.n_kv_heads, head = begin - at * a.n_kv_heads;
  // Its row: the first thread whose sum passes `at`, then that thread's rows in turn.
  int lo = 0, hi = NT - 1;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (before[mid] > at) hi = mid;
    else lo = mid + 1;
  }
  int left = at - (lo ? before[lo - 1] : 0), b = lo * each, first, n;
  while (n = pages_of(b, first), left >= n) left -= n, ++b;
  for (int item = begin;;) {
    const int entry = first + left;
    const int page = __builtin_amdgcn_readfirstlane(a.table[b * a.table_stride + entry]);
    const int held = min(tokens(a.wanted, b) - (entry << a.page_shift), 1 << a.page_shift);
    const bool there = page >= 0 && page < a.n_pages;        // (uniform)
    if (there) {
      const char* src = a.k + page * a.page_stride + head * a.head_stride + 16 * (lane % L);
      Extremes<T> x;
      x.clear();
      for (int t = lane / L; t < held; t += U * (64 / L)) {
        v4u v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)                // (a token twice does no harm)
          v[u] = __builtin_nontemporal_load(
              reinterpret_cast<const v4u*>(src + min(t + u * (64 / L), held - 1) * a.tok_stride));
#pragma unroll
        for (int u = 0; u < U; ++u) x.add(v[u]);
      }
      const bool none = __builtin_amdgcn_ballot_w64(x.bad() && lane / L < held) != 0;
      x.join_rows();
      float most = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) most = fmaxf(most, fmaxf(fabsf(x.largest(i)), fabsf(x.smallest(i))));
      // (over the lanes of a token: rows of 16, and a swap of two rows)
      most = row_max(most);
      if constexpr (L == 32) {
        auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(most), __float_as_uint(most), false, false);
        most = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
      }
      const int e = step_of(none ? 0.f : most);
      const bool wide = none || e > kHighestStep;
      const float up = power_of_two(wide ? 0 : -e);
      // The first row of lanes stores the upper bounds, the second the lower ones.
      if (lane < 2 * L) {
        const bool upper = lane < L;
        int8_t code[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          // (a product that falls below the smallest number still rounds away from 0)
          const float v = upper ? x.largest(i) : -x.smallest(i);
          const float c = v > 0.f ? fmaxf(ceilf(v * up), 1.f) : ceilf(v * up);
          code[i] = wide ? 0 : (int8_t)(upper ? c : -c);
        }
        const int64_t to = (int64_t)page * a.n_kv_heads + head;
        __builtin_memcpy(a.codes + to * kBoundBytes + (upper ? 0 : kD) + N * (lane % L), code, N);
        if (lane == 0) a.scales[to] = wide ? INFINITY : power_of_two(e);
      }
    }
    if (++item == end) return;
    if (++head == a.n_kv_heads) {
      head = 0;
      if (++left == n) {
        left = 0;
        do n = pages_of(++b, first);               // (there are items left: some row has them)
        while (n == 0);
      }
    }
  }
}

// --- scores ---------------------------------------------------------------------------------------

// Keys in the order of the scores: 0 for a page that is not there, kAlways for one picked always.
constexpr uint32_t kAlways = 0xffffffffu;
__device__ inline uint32_t key_of(float score) {
  const uint32_t bits = __float_as_uint(score), key = bits ^ ((int32_t)bits < 0 ? 0xffffffffu : 0x80000000u);
  return min(max(key, 1u), kAlways - 1u);          // (scales that were never set may be any NaN)
}

// Queries of up to 16 heads in 8 bits, as the matrix operand of lane (n, g): head n's channels 16 g ..
// and 64 + 16 g .. , positive parts and then negative parts.
struct Say {
  v4i b[4];
  int e;                                           // the step's exponent, kNoSay: not finite, or no head
};
constexpr int kNoSay = -10000;
__device__ inline Say say_of(const PagedArgs& p, int64_t at, bool on, int g) {
  float x[2][16], top = 0.f;
  bool bad = false;
  const float sign = p.scale < 0.f ? -1.f : 1.f;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    load_queries(p.q, p.q_dtype, at + 64 * u + 16 * g, on, x[u]);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      bad |= !(fabsf(x[u][i]) < INFINITY);
      top = fmaxf(top, fabsf(x[u][i]));
    }
  }
  top = over_groups_max(top);
  bad = over_groups_max(bad ? 1.f : 0.f) > 0.f;
  Say s;
  const int e = step_of(bad ? 0.f : top);
  s.e = on && !bad ? e : kNoSay;
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      uint32_t up = 0u, down = 0u;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float c = x[u][4 * d + i] * power_of_two(-e);
        const int code = bad ? 0 : (int)rintf(sign * c);
        up |= (uint32_t)(max(code, 0) & 0xff) << 8 * i;
        down |= (uint32_t)(min(code, 0) & 0xff) << 8 * i;
      }
      s.b[u][d] = (int)up;
      s.b[2 + u][d] = (int)down;
    }
  return s;
}

// A workgroup of four waves scores 64 R pages of a (sequence, KV head), a wave 16 of them at a time.
// Reads 260 bytes a page: the memory bounds it, or the latency of three loads in series (the length with
// entries and queries, bounds).  ONE: at most 16 query heads a KV head, in registers; else in LDS.
template <bool ONE, int R>
__global__ __launch_bounds__(256) void score_kernel(SparseArgs a) {
  constexpr int HG = ONE ? 1 : kMaxSay / 16, kChunk = 64 * R;
  __shared__ v4i ops[ONE ? 1 : HG][4][64];
  __shared__ int exps[HG][16];
  const PagedArgs& p = a.p;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int chunks = (p.max_pages + kChunk - 1) / kChunk;
  const int row = (int)blockIdx.x / chunks, chunk = (int)blockIdx.x % chunks;
  const int seq = row / p.n_kv_heads, kvh = row % p.n_kv_heads;

  // The wave's tiles of pages: entries (of all there are, before the length is known), then bounds.
  const int base = chunk * kChunk + wave * 16 * R;
  int page[R];
#pragma unroll
  for (int r = 0; r < R; ++r)
    page[r] = p.table[seq * p.table_stride + min(base + 16 * r + n, p.max_pages - 1)];
  const int len = min(max(p.seq_len[seq], 0), p.len_max);
  const int pages = (len + (1 << p.page_shift) - 1) >> p.page_shift;
  if (pages <= a.most || chunk * kChunk >= pages) return;      // (all are picked; none here)
#pragma unroll
  for (int r = 0; r < R; ++r)
    page[r] = base + 16 * r + n < pages && page[r] < p.n_pages ? page[r] : -1;
  v4i x[R][4];
  float scale[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t at = (int64_t)max(page[r], 0) * p.n_kv_heads + kvh;
#pragma unroll
    for (int s = 0; s < 4; ++s)
      x[r][s] = *reinterpret_cast<const v4i*>(a.codes + at * kBoundBytes + 64 * s + 16 * g);
    scale[r] = a.scales[at];
  }

  const int64_t q_row = seq * p.q_stride + (int64_t)kvh * p.G * kD;
  Say say;
  int top_e;
  if constexpr (ONE) {
    say = say_of(p, q_row + (int64_t)min(n, p.G - 1) * kD, n < p.G, g);
    top_e = say.e;
  } else {
    top_e = kNoSay;
    for (int h = wave; h < p.hg; h += 4) {
      const int head = 16 * h + n;
      say = say_of(p, q_row + (int64_t)min(head, p.G - 1) * kD, head < p.G, g);
#pragma unroll
      for (int s = 0; s < 4; ++s) ops[h][s][lane] = say.b[s];
      if (g == 0) exps[h][n] = say.e;
    }
    __syncthreads();
    for (int h = 0; h < p.hg; ++h) top_e = max(top_e, exps[h][n]);
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) top_e = max(top_e, __shfl_xor(top_e, o, 64));

#pragma unroll
  for (int r = 0; r < R; ++r) {
    float best[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    for (int h = 0; h < (ONE ? 1 : p.hg); ++h) {
      v4i sum = {0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < 4; ++s)
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[r][s], ONE ? say.b[s] : ops[ONE ? 0 : h][s][lane],
                                                    sum, 0, 0, 0);
      const int e = ONE ? say.e : exps[ONE ? 0 : h][n];
      const float w = power_of_two(max(e - top_e, -60));
#pragma unroll
      for (int i = 0; i < 4; ++i) best[i] = e == kNoSay ? best[i] : fmaxf(best[i], (float)sum[i] * w);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) best[i] = row_max(best[i]);
    // Lane (n, g), n < 4, has page 4 g + n of the tile.
    const float mine = n == 0 ? best[0] : n == 1 ? best[1] : n == 2 ? best[2] : best[3];
    const int from = (lane & 48) | ((4 * g + n) & 15);
    const float steps = __shfl(scale[r], from, 64);
    const bool there = __shfl(page[r], from, 64) >= 0;
    const int i = base + 16 * r + 4 * g + n;
    if (n < 4 && i < pages) {
      const float score = steps == INFINITY ? INFINITY : mine == -INFINITY ? 0.f : mine * steps;
      const bool always = i < a.first || i >= pages - a.last;
      a.keys[row * a.key_stride + i] = !there ? 0u : always ? kAlways : key_of(score);
    }
  }
}

// --- the choice, and attention --------------------------------------------------------------------

constexpr int kSparseWaves = 8, kSparseGroups = 256, kSparseCounterStride = 64;
constexpr size_t kSparseCountersBytes = (size_t)kSparseGroups * kSparseCounterStride * sizeof(unsigned);
constexpr int kHeldKeys = 16;                      // keys of a thread in registers
constexpr int kBins = 1024;                        // of a pass of the choice: 10 bits of the keys
constexpr int kListed = 2048;                      // picked pages of a workgroup in LDS

// A row (a sequence, a KV head, up to 16 of its query heads) has `parts` workgroups.  Each of them finds
// the row's pages for itself, which takes no longer than to wait for another that does, and attends its
// share of them with the tile of paged_tile.h; the last one joins the parts.
template <class M, int QT>
__global__ __launch_bounds__(64 * kSparseWaves, 2) void sparse_kernel(SparseArgs a) {
  constexpr int W = kSparseWaves, NT = 64 * W, TT = M::kTokens, NM = M::kMine;
  __shared__ JoinSpace<W, kSparseGroups> sh;
  __shared__ int list_entry[kListed], list_page[kListed];
  __shared__ int hist[2][kBins], sums[5][W], found[3];
  __shared__ unsigned arrived;
  const PagedArgs& p = a.p;
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = (int)blockIdx.x / a.parts, part = (int)blockIdx.x % a.parts;
  const int pair = row / p.hg, hgi = row % p.hg;   // (sequence, KV head)
  const int seq = pair / p.n_kv_heads, kvh = pair % p.n_kv_heads;
  const int len = min(max(p.seq_len[seq], 0), p.len_max);
  const int shift = p.page_shift;
  const int pages = (len + (1 << shift) - 1) >> shift;
  const int32_t* table = p.table + seq * p.table_stride;
  const uint32_t* keys = a.keys + pair * a.key_stride;
  auto exists = [&](int page) { return (page >= 0) & (page < p.n_pages); };

  // Queries early: their loads take as long as the choice.
  const int heads = min(kPagedHeads, p.G - hgi * kPagedHeads);
  typename M::template Query<QT> q;
  q.load(p.q, p.q_dtype,
         seq * p.q_stride + ((int64_t)kvh * p.G + hgi * kPagedHeads + min(n, heads - 1)) * kD,
         n < heads, g);

  // Thread t has the keys of `run` pages from t run on: a multiple of four in registers, or any
  // number that is read again each time.
  const bool all = pages <= a.most;                // (then there are no keys)
  const bool fits = pages <= kHeldKeys * NT;
  const int run = fits ? (pages + 4 * NT - 1) / (4 * NT) * 4 : (pages + NT - 1) / NT, mine0 = tid * run;
  auto key_at = [&](int i) -> uint32_t {
    return i >= pages ? 0u : all ? (exists(table[i]) ? kAlways : 0u) : keys[i];
  };
  uint32_t held[kHeldKeys];
#pragma unroll
  for (int r = 0; r < kHeldKeys; r += 4) {
    v4u k = {0u, 0u, 0u, 0u};
    if (fits && r < run) {                         // (uniform)
      if (!all && mine0 + r + 4 <= pages) {
        k = *reinterpret_cast<const v4u*>(keys + mine0 + r);
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u) k[u] = key_at(mine0 + r + u);
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) held[r + u] = k[u];
  }
  auto each_key = [&](auto f) {
    if (fits) {
#pragma unroll
      for (int r = 0; r < kHeldKeys; r += 4) {
        if (r >= run) break;                       // (uniform)
#pragma unroll
        for (int u = 0; u < 4; ++u) f(held[r + u], mine0 + r + u);
      }
    } else {
      for (int r = 0; r < run; ++r) f(key_at(mine0 + r), mine0 + r);
    }
  };
  // Pages are picked whose key is above `limit`, and the first `ties` of those with that key.  The
  // limit is found by counting the keys in bins of a range that holds it, which the next pass divides.
  uint32_t limit = 0u;
  int ties = 0;
  if (!all) {
    uint32_t least = kAlways, top = 0u;            // of the keys that are to be compared
    int there = 0, always = 0;
    each_key([&](uint32_t k, int) {
      there += k != 0u;
      always += k == kAlways;
      const bool normal = k != 0u && k != kAlways;
      least = normal ? min(least, k) : least;
      top = normal ? max(top, k) : top;
    });
    there = wave_scan_sum(there);
    always = wave_scan_sum(always);
    least = (uint32_t)wave_scan((int)least, -1, [](int x, int y) { return (int)min((uint32_t)x, (uint32_t)y); });
    top = (uint32_t)wave_scan((int)top, 0, [](int x, int y) { return (int)max((uint32_t)x, (uint32_t)y); });
    if (lane == 63) {
      hist[0][wave] = (int)least;
      hist[0][W + wave] = (int)top;
      sums[1][wave] = there;
      sums[2][wave] = always;
    }
    __syncthreads();
    there = always = 0;
    least = kAlways;
    top = 0u;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      there += sums[1][w];
      always += sums[2][w];
      least = min(least, (uint32_t)hist[0][w]);
      top = max(top, (uint32_t)hist[0][W + w]);
    }
    there = __builtin_amdgcn_readfirstlane(there);
    int need = a.most - __builtin_amdgcn_readfirstlane(always);
    if (there > a.most) {
      if (need == 0) {
        limit = kAlways - 1u;
      } else {
        uint32_t from = __builtin_amdgcn_readfirstlane(least);
        int bits = 32 - __clz((int)(__builtin_amdgcn_readfirstlane(top) - from));   // of the range
        __syncthreads();                           // (the bins are read)
        for (int i = tid; i < 2 * kBins; i += NT) hist[0][i] = 0;
        __syncthreads();
        for (int turn = 0;; turn ^= 1) {
          const int shift_by = max(bits - 10, 0);
          const uint32_t in_range = 1u << (bits - shift_by);           // (keys behind it count no more)
          int* bins = hist[turn];
          each_key([&](uint32_t k, int) {
            const uint32_t bin = (k - from) >> shift_by;
            if (k != kAlways && k >= from && bin < in_range) atomicAdd(&bins[bin], 1);
          });
          __syncthreads();
          // From the highest bin down, two a thread.
          const int c0 = bins[kBins - 1 - 2 * tid], c1 = bins[kBins - 2 - 2 * tid];
          static_assert(kBins == 2 * NT, "two bins a thread");
          int incl = wave_scan_sum(c0 + c1);
          if (lane == 63) sums[0][wave] = incl;
          __syncthreads();
#pragma unroll
          for (int w = 0; w < W; ++w) incl += w < wave ? sums[0][w] : 0;
          const int before = incl - c0 - c1;
          if (before < need && need <= incl) {     // (one thread)
            const bool second = need > before + c0;
            found[0] = kBins - 1 - 2 * tid - (second ? 1 : 0);
            found[1] = second ? before + c0 : before;
            found[2] = second ? c1 : c0;
          }
          bins[kBins - 1 - 2 * tid] = bins[kBins - 2 - 2 * tid] = 0;
          __syncthreads();
          from += (uint32_t)__builtin_amdgcn_readfirstlane(found[0]) << shift_by;
          need -= __builtin_amdgcn_readfirstlane(found[1]);
          if (need == __builtin_amdgcn_readfirstlane(found[2])) {      // all of the bin
            limit = from - 1u;
            break;
          }
          if (shift_by == 0) {
            limit = from;
            ties = need;
            break;
          }
          bits = shift_by;
        }
      }
    }
  }

  // The picked pages in order: each part keeps its own and those are told.
  const int first = part * a.run;                  // tiles
  const int from = (int)((int64_t)first * TT >> shift);
  const int until = (int)(((int64_t)(first + a.run) * TT + (1 << shift) - 1) >> shift);
  int gt = 0, eq = 0;
  each_key([&](uint32_t k, int) {
    gt += k > limit;
    eq += ties && k == limit;
  });
  int gt_before = wave_scan_sum(gt), eq_before = wave_scan_sum(eq);
  if (lane == 63) {                                // (rows of their own: other waves may still read the others)
    sums[3][wave] = gt_before;
    sums[4][wave] = eq_before;
  }
  __syncthreads();
  int gt_all = 0, eq_all = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const int x = sums[3][w], y = sums[4][w];
    gt_before += w < wave ? x : 0;
    eq_before += w < wave ? y : 0;
    gt_all += x;
    eq_all += y;
  }
  gt_before -= gt;
  eq_before -= eq;
  if (gt + eq > 0)
    each_key([&](uint32_t k, int i) {
      const bool above = k > limit, tie = ties && k == limit;
      const int pos = gt_before + min(eq_before, ties);
      if ((above || (tie && eq_before < ties)) && pos >= from && pos < until) {
        if (pos - from < kListed) list_entry[pos - from] = i;
        else a.picked[(int64_t)pair * a.most + pos] = i;     // (the same by every reader of it)
      }
      gt_before += above;
      eq_before += tie;
    });
  const int picked = __builtin_amdgcn_readfirstlane(gt_all) + min(__builtin_amdgcn_readfirstlane(eq_all), ties);
  const int tiles = (int)(((int64_t)picked << shift) + TT - 1) / TT;
  const int parts = max(1, (tiles + a.run - 1) / a.run);
  if (part >= parts) return;                       // (uniform)
  if (part == 0 && hgi == 0)
    for (int i = picked + tid; i < a.most; i += NT) a.picked[(int64_t)pair * a.most + i] = -1;
  __syncthreads();
  for (int j = tid; j < min(min(until, picked) - from, kListed); j += NT) {
    const int i = list_entry[j];
    list_page[j] = table[i];
    a.picked[(int64_t)pair * a.most + from + j] = i;
  }
  __syncthreads();

  // Attention over the picked pages' tokens, as if they were one sequence: token v of it.
  const int last = min(first + a.run, tiles);
  struct Place {
    int page, token;                               // (-1: no page); the first token's index
  };
  auto place = [&](int v) {
    const int j = v >> shift;
    Place w{-1, 0};
    if (j < picked) {
      int entry;
      if (j - from < kListed) {
        entry = list_entry[j - from];
        w.page = list_page[j - from];
      } else {
        entry = a.picked[(int64_t)pair * a.most + j];
        w.page = table[entry];
      }
      w.token = (entry << shift) + (v & ((1 << shift) - 1));
    }
    return w;
  };
  typename M::Keys key;
  typename M::Values val;
  auto slot_of = [&](const Place& w) {
    return kvh * p.head_stride + max(w.page, 0) * p.page_stride +
           (w.token & ((1 << shift) - 1)) * p.tok_stride;
  };
  auto load_keys = [&](int t0) {
    const int v = t0 + M::key_token(0, n);
    key.load(p.k + slot_of(place(v)), p.tok_stride, g);
  };
  RowPart mine;
  v4f(&acc)[8] = mine.acc;
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = (v4f){0.f, 0.f, 0.f, 0.f};
  float m_run = -INFINITY, l_run = 0.f;
  bool seen = false;
  Place at{-1, 0};
  if (first + wave < last) {
    load_keys((first + wave) * TT);
    at = place((first + wave) * TT + NM * g);
    val.load(p.v + slot_of(at), p.tok_stride, n);
  }
  for (int i = first + wave; i < last; i += W) {
    const bool more = i + W < last;
    float z[NM];
    M::template scores<QT>(key, q, z);
    if (more) load_keys((i + W) * TT);
    const Place next = place(min(i + W, last - 1) * TT + NM * g);
    if (p.cap > 0.f) {
      const float in = p.scale / p.cap, back = p.cap * kLog2e;
#pragma unroll
      for (int e = 0; e < NM; ++e) z[e] = back * tanh_of(z[e] * in);
    } else {
#pragma unroll
      for (int e = 0; e < NM; ++e) z[e] *= p.scale * kLog2e;
    }
    if (__builtin_amdgcn_ballot_w64((at.page < 0) | (at.token + NM > len))) {
      bool any = false;
#pragma unroll
      for (int e = 0; e < NM; ++e) {
        const bool on = (at.page >= 0) & (at.token + e < len);
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
    const float sa = __builtin_amdgcn_exp2f(m_run - ref);      // (0 at the first tile)
    float w[NM], sum = 0.f;
#pragma unroll
    for (int e = 0; e < NM; ++e) {
      w[e] = __builtin_amdgcn_exp2f(z[e] - ref);
      sum += w[e];
    }
    l_run = l_run * sa + sum;
    m_run = m;
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] *= sa;
    M::accumulate(val, w, acc);
    if (more) val.load(p.v + slot_of(next), p.tok_stride, n);
    at = next;
  }
  mine.m = m_run;
  mine.l = over_groups_sum(l_run);
  if (seen && mine.m == -INFINITY && mine.l == 0.f) {          // (NaN scores: the sum is NaN)
    mine.m = kLowest;
    mine.l = 1.f;
  }

  // The waves' parts meet in LDS, the workgroups' in the workspace.
  if (g == 0) {
    sh.m[wave][n] = mine.m;
    sh.l[wave][n] = mine.l;
  }
  if (n < heads) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) sh.sums[wave][n][M::channel(j, i, g)] = acc[j][i];
  }
  __syncthreads();
  const int64_t q_row = (int64_t)seq * p.n_q_heads + kvh * p.G + hgi * kPagedHeads;
  const auto slots = __builtin_amdgcn_make_buffer_rsrc(p.parts, (short)0, p.parts_bytes, kRsrcWord3);
  auto finish = [&](int h, int c4, float m, float l, v4f o) {
    finish_row(p, q_row + h, c4, m, l, o);
  };
  auto part_at = [&](int x, int h) {
    return ((row * a.parts + x) * p.slot_heads + h) * (int)sizeof(Partial);
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
        __builtin_amdgcn_raw_buffer_store_b128((v4i)(v4f){m, l, 0.f, 0.f}, slots, off, 0, kCoherent);
    }
  }
  if (parts == 1) return;
  unsigned* counter = p.counters + row * kSparseCounterStride;
  __builtin_amdgcn_s_waitcnt(0);                   // this thread's stores are done
  __syncthreads();
  if (tid == 0)
    arrived = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (arrived != (unsigned)parts - 1u) return;
  join_parts(sh, parts, heads, finish, [&](int x, int h, int off) {
    return (v4f)__builtin_amdgcn_raw_buffer_load_b128(slots, part_at(x, h) + off, 0, kCoherent);
  });
  if (tid == 0) *counter = 0u;                     // as the next call expects it
}

// Rows of keys begin at 16 bytes.
int64_t key_stride_of(int64_t max_pages) { return (max_pages + 3) / 4 * 4; }

// Rows, and part slots: rows that are shared are so by no more workgroups than fill the chip.
int64_t sparse_rows(int64_t batch, int n_q_heads, int n_kv_heads) {
  const int G = n_q_heads / n_kv_heads;
  return batch * n_kv_heads * ((G + kPagedHeads - 1) / kPagedHeads);
}
size_t sparse_parts_bytes(int slot_heads) {
  return (size_t)kSparseGroups * slot_heads * sizeof(Partial);
}
int slot_heads_of(int n_q_heads, int n_kv_heads) {
  return std::min(n_q_heads / n_kv_heads, kPagedHeads);
}

}  // namespace

aatc_status launch_bounds(const BoundsArgs& a, aatc_dtype dtype, void* stream) {
  const int64_t items = (int64_t)a.rows * a.max_pages * a.n_kv_heads;
  const int64_t grid = std::min<int64_t>(kBoundGroups, (items + kBoundWaves - 1) / kBoundWaves);
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * kBoundWaves), 0, (hipStream_t)stream,
                       a);
    return hipGetLastError() == hipSuccess ? AATC_OK : AATC_E_DEVICE;
  };
  switch (dtype) {
    case AATC_F32: return launch(bounds_kernel<float>);
    case AATC_BF16: return launch(bounds_kernel<__bf16>);
    default: return launch(bounds_kernel<_Float16>);
  }
}

size_t sparse_workspace_bytes(int batch, int n_q_heads, int n_kv_heads, int64_t max_pages) {
  return kSparseCountersBytes + round256(sparse_parts_bytes(slot_heads_of(n_q_heads, n_kv_heads))) +
         (size_t)batch * n_kv_heads * key_stride_of(max_pages) * sizeof(uint32_t);
}

bool sparse_fits(int64_t batch, int n_q_heads, int n_kv_heads, int64_t max_pages) {
  if (n_q_heads / n_kv_heads > kMaxSay) return false;
  const int64_t pairs = batch * n_kv_heads;
  if (max_pages > ((int64_t)1 << 30) / pairs) return false;
  return pairs * ((max_pages + 63) / 64) <= kMaxSparseGroups &&
         sparse_rows(batch, n_q_heads, n_kv_heads) <= kMaxSparseGroups;
}

aatc_status launch_sparse(SparseArgs a, aatc_dtype c_dtype, void* workspace, void* stream) {
  PagedArgs& p = a.p;
  p.slot_heads = slot_heads_of(p.n_q_heads, p.n_kv_heads);
  p.len_max = std::min(p.len_max, INT32_MAX - 16384);          // (tokens of whole tiles: 32 bits)
  p.counters = static_cast<unsigned*>(workspace);
  char* parts = static_cast<char*>(workspace) + kSparseCountersBytes;
  p.parts = reinterpret_cast<Partial*>(parts);
  p.parts_bytes = (int)sparse_parts_bytes(p.slot_heads);
  a.keys = reinterpret_cast<uint32_t*>(parts + round256(p.parts_bytes));
  a.key_stride = key_stride_of(p.max_pages);
  const int tt = c_dtype == AATC_F32 ? Full32<false>::kTokens : Half16<__bf16, false>::kTokens;
  const int64_t rows = sparse_rows(p.batch, p.n_q_heads, p.n_kv_heads);
  const int64_t tokens = (int64_t)std::min(a.most, p.max_pages) << p.page_shift;
  const int tiles = (int)((tokens + tt - 1) / tt);
  // Rows are shared where there are fewer than workgroups, a tile a wave at least.
  const int share = rows < kSparseGroups ? kSparseGroups / (int)rows : 1;
  a.run = std::max((tiles + share - 1) / share, std::min(tiles, kSparseWaves));
  a.parts = (tiles + a.run - 1) / a.run;
  const hipStream_t st = (hipStream_t)stream;
  if (p.max_pages > a.most) {                      // (else every page is picked)
    // Few pages in small chunks, for the chip's sake; many in large ones, whose queries' codes count less.
    const int64_t pairs = (int64_t)p.batch * p.n_kv_heads;
    const bool many = pairs * p.max_pages >= 256 * 1024;
    const int chunk = many || p.hg > 1 ? 256 : 64;
    const dim3 groups((unsigned)(pairs * ((p.max_pages + chunk - 1) / chunk)));
    if (p.hg > 1)
      hipLaunchKernelGGL((score_kernel<false, 4>), groups, dim3(256), 0, st, a);
    else if (many)
      hipLaunchKernelGGL((score_kernel<true, 4>), groups, dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL((score_kernel<true, 1>), groups, dim3(256), 0, st, a);
    if (hipGetLastError() != hipSuccess) return AATC_E_DEVICE;
  }
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)(rows * a.parts)), dim3(64 * kSparseWaves), 0, st, a);
    return hipGetLastError() == hipSuccess ? AATC_OK : AATC_E_DEVICE;
  };
  using One = std::integral_constant<int, 1>;
  using Three = std::integral_constant<int, 3>;
  const bool same = p.q_dtype == (int)c_dtype;
  auto launch_as = [&](auto m, auto qt) {
    return launch(sparse_kernel<decltype(m), decltype(qt)::value>);
  };
  switch (c_dtype) {
    case AATC_F32: return launch_as(Full32<false>{}, One{});
    case AATC_BF16:
      return same ? launch_as(Half16<__bf16, false>{}, One{})
                  : launch_as(Half16<__bf16, false>{}, Three{});
    default:
      return same ? launch_as(Half16<_Float16, false>{}, One{})
                  : launch_as(Half16<_Float16, false>{}, Three{});
  }
}

}  // namespace aatc
