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
// The tiles of all rows (sequence, KV head, 16 query heads) lie in one line that the workgroups
// share evenly, whatever the lengths.  A row that several workgroups share is joined by the last
// of them to arrive, in the order of the parts.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <algorithm>

#include "paged.h"
#include "paged_plan.h"
#include "params.h"

namespace aatc {
namespace {

constexpr int kPagedThreads = 256, kPagedWaves = kPagedThreads / 64;
constexpr int kPagedGroups = 512;                 // most workgroups: two per compute unit
constexpr int kPagedHeads = 16;                   // query heads of a row
constexpr int kQuotaMin = kPagedWaves;            // tiles of a workgroup: one per wave at least
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kPartFloats = kPagedHeads * (kD + 2);   // m [16], l [16], o [16][128]
constexpr int kRowStride = 64;                    // counters 256 bytes apart (their atomics
                                                  // would queue on one cache line)

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Lane l with lane l ^ 16, l ^ 32.
__device__ inline float over_groups_max(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float over_groups_sum(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Stores and loads of workspace that other workgroups write: performed where every compute
// unit of the device sees them.
__device__ inline void st_dev(float* p, float v) {
  __hip_atomic_store(reinterpret_cast<unsigned*>(p), __float_as_uint(v), __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline float ld_dev(const float* p) {
  return __uint_as_float(__hip_atomic_load(reinterpret_cast<const unsigned*>(p), __ATOMIC_RELAXED,
                                           __HIP_MEMORY_SCOPE_AGENT));
}

// N consecutive query elements from element i on (aligned to the element only).
template <class T, int N>
struct Run {
  T e[N];
};
template <int N>
__device__ inline void load_queries(const void* q, int dtype, int64_t i, bool on, float (&x)[N]) {
  Run<float, N> f;
  Run<__bf16, N> b;
  Run<_Float16, N> h;
  if (dtype == AATC_F32) __builtin_memcpy(&f, static_cast<const float*>(q) + i, sizeof f);
  else if (dtype == AATC_BF16) __builtin_memcpy(&b, static_cast<const __bf16*>(q) + i, sizeof b);
  else __builtin_memcpy(&h, static_cast<const _Float16*>(q) + i, sizeof h);
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const float v = dtype == AATC_F32 ? f.e[e] : dtype == AATC_BF16 ? (float)b.e[e] : (float)h.e[e];
    x[e] = on ? v : 0.f;
  }
}

// The two products on 16-bit types.  A lane's place: n = lane % 16, g = lane / 16.
template <class T>
struct Half16 {
  static constexpr bool kF16 = sizeof(T) == 2 && __is_same(T, _Float16);
  typedef T v8 __attribute__((ext_vector_type(8)));
  static constexpr int kTokens = 32;              // of a tile
  static constexpr int kMine = 8;                 // scores of a lane: tokens 8 g .. 8 g + 7
  static constexpr int kTerms = kF16 ? 2 : 3;     // of P
  static constexpr float kLower = kF16 ? 14.f : 0.f;
  // Token of the tile whose key chunk u (of two) lane (n, g) loads, and the 8-token block that
  // a lane's keys and values are in.
  static __device__ int key_token(int u, int n) { return 8 * (n >> 2) + 4 * u + (n & 3); }
  static __device__ int key_block(int n) { return n >> 2; }
  static __device__ int value_block(int g) { return g; }

  static __device__ v4f mfma(v8 a, v8 b, v4f c) {
    if constexpr (kF16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }

  // Queries as terms: lane (n, g) holds head n's channels 8 (4 kk + g) .. + 7.
  template <int QT>
  struct Query {
    v8 t[QT][4];
    float back;                                   // head n's scores times this
    __device__ void load(const void* q, int dtype, int64_t at, bool on, int g) {
      if constexpr (QT == 1) {
        back = 1.f;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          v4u x;
          __builtin_memcpy(&x, static_cast<const T*>(q) + at + 8 * (4 * kk + g), 16);
          t[0][kk] = __builtin_bit_cast(v8, on ? x : (v4u){0u, 0u, 0u, 0u});
        }
      } else {
        float x[4][8], top = 0.f;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          load_queries(q, dtype, at + 8 * (4 * kk + g), on, x[kk]);
#pragma unroll
          for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[kk][e]));
        }
        // f16 holds the terms of a head whose largest channel is near 2^15, down to 2^-39 of it.
        int up = 0;
        if constexpr (kF16) {
          top = over_groups_max(top);
          if (top > 0.f && top < INFINITY) up = 14 - ilogbf(top);
          up = max(-126, min(126, up));
        }
        back = ldexpf(1.f, -up);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float r = kF16 ? ldexpf(x[kk][e], up) : x[kk][e];
#pragma unroll
            for (int i = 0; i < QT; ++i) {
              t[i][kk][e] = (T)r;
              r -= (float)t[i][kk][e];
            }
          }
      }
    }
  };

  struct Keys {
    v4u r[2][4];
    // row(u): the lane's row of chunk u
    __device__ void load(const char* row0, int64_t tok_stride, int g) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          r[u][kk] = *reinterpret_cast<const v4u*>(row0 + u * 4 * tok_stride + 64 * kk + 16 * g);
    }
  };
  struct Values {
    v4u r[8];
    __device__ void load(const char* row0, int64_t tok_stride, int n) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        r[e] = *reinterpret_cast<const v4u*>(row0 + e * tok_stride + 16 * n);
    }
    // Token e of the lane's counts as zeros unless `on` (0 times what is stored there may be NaN).
    __device__ void keep(int e, bool on) {
#pragma unroll
      for (int i = 0; i < 4; ++i) r[e][i] = on ? r[e][i] : 0u;
    }
  };

  template <int QT>
  static __device__ void scores(const Keys& k, const Query<QT>& q, float (&z)[kMine]) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      v4f s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = QT - 1; i >= 0; --i)
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          s = mfma(__builtin_bit_cast(v8, k.r[u][kk]), q.t[i][kk], s);
#pragma unroll
      for (int i = 0; i < 4; ++i) z[4 * u + i] = s[i] * q.back;
    }
  }

  // acc[j][i]: channel 8 (4 g + i) + j of head n.
  static __device__ int channel(int j, int i, int g) { return 8 * (4 * g + i) + j; }
  static __device__ void accumulate(const Values& v, const float (&p)[kMine], v4f (&acc)[8]) {
    v8 t[kTerms];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float r = p[e];
#pragma unroll
      for (int i = 0; i < kTerms; ++i) {
        t[i][e] = (T)r;
        r -= (float)t[i][e];
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v4u a;                                      // column j of the lane's 8 x 8 block
#pragma unroll
      for (int d = 0; d < 4; ++d)
        a[d] = __builtin_amdgcn_perm(v.r[2 * d + 1][j / 2], v.r[2 * d][j / 2],
                                     j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int i = kTerms - 1; i >= 0; --i) acc[j] = mfma(__builtin_bit_cast(v8, a), t[i], acc[j]);
    }
  }
};

// The two products on float32 (v_mfma_f32_16x16x4_f32: no splitting).
struct Full32 {
  static constexpr int kTokens = 16;
  static constexpr int kMine = 4;                 // tokens 4 g .. 4 g + 3
  static constexpr float kLower = 0.f;
  static __device__ int key_token(int, int n) { return n; }
  static __device__ int key_block(int n) { return n >> 3; }
  static __device__ int value_block(int g) { return g >> 1; }
  static __device__ v4f mfma(float a, float b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
  }
  template <int QT>
  struct Query {                                  // channels 16 c + 4 g .. + 3
    v4f t[8];
    __device__ void load(const void* q, int dtype, int64_t at, bool on, int g) {
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        float x[4];
        load_queries(q, dtype, at + 16 * c + 4 * g, on, x);
        t[c] = (v4f){x[0], x[1], x[2], x[3]};
      }
    }
  };
  struct Keys {
    v4f r[8];
    __device__ void load(const char* row0, int64_t, int g) {
#pragma unroll
      for (int c = 0; c < 8; ++c) r[c] = *reinterpret_cast<const v4f*>(row0 + 64 * c + 16 * g);
    }
  };
  struct Values {
    v4f r[4][2];
    __device__ void load(const char* row0, int64_t tok_stride, int n) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < 2; ++c)
          r[e][c] = *reinterpret_cast<const v4f*>(row0 + e * tok_stride + 256 * c + 16 * n);
    }
    __device__ void keep(int e, bool on) {
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) r[e][c][i] = on ? r[e][c][i] : 0.f;
    }
  };
  template <int QT>
  static __device__ void scores(const Keys& k, const Query<QT>& q, float (&z)[kMine]) {
    v4f s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 8; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) s = mfma(k.r[c][e], q.t[c][e], s);
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = s[i];
  }
  // acc[4 c + e][i]: channel 64 c + 4 (4 g + i) + e of head n.
  static __device__ int channel(int j, int i, int g) {
    return 64 * (j >> 2) + 4 * (4 * g + i) + (j & 3);
  }
  static __device__ void accumulate(const Values& v, const float (&p)[kMine], v4f (&acc)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[4 * c + e] = mfma(v.r[i][c][e], p[i], acc[4 * c + e]);
  }
};

template <class M, int QT>
__global__ __launch_bounds__(kPagedThreads) void paged_kernel(PagedArgs a) {
  constexpr int TT = M::kTokens, NM = M::kMine;
  constexpr int kOs = kD + 4;                      // LDS row of a head's sums (banks)
  __shared__ float so[kPagedWaves][kPagedHeads][kOs];
  __shared__ float sm[kPagedWaves][kPagedHeads], sl[kPagedWaves][kPagedHeads];
  __shared__ int scan[kPagedWaves], found[2];
  __shared__ unsigned arrived;
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rows = a.n_kv_heads * a.hg;            // of a sequence

  auto tiles_of = [&](int b) {
    const int len = min(max(a.seq_len[b], 0), a.len_max);
    return row_tiles(len, a.window, a.sink, TT);
  };

  // The line: every thread adds up a run of sequences, a scan over the workgroup.
  const int each = (a.batch + kPagedThreads - 1) / kPagedThreads;
  const int b0 = min(tid * each, a.batch), b1 = min(b0 + each, a.batch);
  int mine = 0;
  for (int b = b0; b < b1; ++b) mine += tiles_of(b).n * rows;
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(incl, o, 64);
    incl += lane >= o ? up : 0;
  }
  if (lane == 63) scan[wave] = incl;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int w = 0; w < kPagedWaves; ++w) {
    incl += w < wave ? scan[w] : 0;
    total += scan[w];
  }
  const int quota = max(kQuotaMin, (total + (int)gridDim.x - 1) / (int)gridDim.x);
  const int begin = (int)blockIdx.x * quota;
  if (begin >= total) return;                      // (uniform)
  const int end = min(begin + quota, total);
  int at = incl - mine;
  if (begin >= at && begin < incl) {               // (one thread: runs without tiles are empty)
    int b = b0;
    for (;; ++b) {
      const int t = tiles_of(b).n * rows;
      if (begin < at + t) break;
      at += t;
    }
    found[0] = b;
    found[1] = at;
  }
  __syncthreads();
  int seq = __builtin_amdgcn_readfirstlane(found[0]);
  const int before = __builtin_amdgcn_readfirstlane(found[1]);
  RowTiles rt = tiles_of(seq);
  int row = (begin - before) / rt.n;               // of the sequence
  int start = before + row * rt.n;               // the row's first tile in the line

  for (;;) {
    const int len = min(max(a.seq_len[seq], 0), a.len_max);
    const int lo = a.window > 0 ? max(0, len - a.window) : 0;
    const int kvh = row / a.hg, h0 = kvh * a.G + (row % a.hg) * kPagedHeads;
    const int heads = min(kPagedHeads, (kvh + 1) * a.G - h0);
    const int64_t q_row = (int64_t)seq * a.n_q_heads + h0;
    const int first = max(begin, start) - start, last = min(end, start + rt.n) - start;
    const int32_t* table = a.table + seq * a.table_stride;
    const char* kb = a.k + kvh * a.head_stride;
    const char* vb = a.v + kvh * a.head_stride;

    typename M::template Query<QT> q;
    q.load(a.q, a.q_dtype, (int64_t)seq * a.q_stride + (int64_t)(h0 + min(n, heads - 1)) * kD,
           n < heads, g);
    const float slope = a.slopes && n < heads ? a.slopes[h0 + n] * kLog2e : 0.f;

    float m_run = -INFINITY, l_run = 0.f;
    v4f acc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = (v4f){0.f, 0.f, 0.f, 0.f};

    // Page of the 8-token block `blk` of the tile at token t0 (-1: none there).
    auto page_of = [&](int t0, int blk) {
      const int i = (t0 + 8 * blk) >> a.page_shift;
      return i < a.max_pages ? table[i] : -1;
    };
    const int slot_mask = (1 << a.page_shift) - 1;
    auto key_row = [&](int t0, int page) {
      const int t = t0 + M::key_token(0, n);
      return kb + max(page, 0) * a.page_stride + (t & slot_mask) * a.tok_stride;
    };
    auto value_row = [&](int t0, int page) {
      const int t = t0 + NM * g;
      return vb + max(page, 0) * a.page_stride + (t & slot_mask) * a.tok_stride;
    };
    auto checked = [&](int page) { return page >= 0 && page < a.n_pages ? page : -1; };

    typename M::Keys key;
    typename M::Values val;
    int i = first + wave;
    int t0 = 0, vp = -1;
    if (i < last) {
      t0 = rt.token(i, TT);
      const int kp = checked(page_of(t0, M::key_block(n)));
      vp = checked(page_of(t0, M::value_block(g)));
      key.load(key_row(t0, kp), a.tok_stride, g);
      val.load(value_row(t0, vp), a.tok_stride, n);
    }
    while (i < last) {
      const int in = i + kPagedWaves;
      const bool more = in < last;
      const int tn = more ? rt.token(in, TT) : t0;
      int kpn = -1, vpn = -1;
      if (more) {
        kpn = checked(page_of(tn, M::key_block(n)));
        vpn = checked(page_of(tn, M::value_block(g)));
      }
      float z[NM];
      M::template scores<QT>(key, q, z);
      if (more) key.load(key_row(tn, kpn), a.tok_stride, g);
      if (a.cap > 0.f) {
#pragma unroll
        for (int e = 0; e < NM; ++e) z[e] = a.cap * tanhf(z[e] * a.scale / a.cap) * kLog2e;
      } else {
#pragma unroll
        for (int e = 0; e < NM; ++e) z[e] *= a.scale * kLog2e;
      }
      if (a.slopes) {
#pragma unroll
        for (int e = 0; e < NM; ++e) z[e] -= slope * (float)(len - 1 - (t0 + NM * g + e));
      }
      // A tile that is attended as a whole needs no masks.
      const bool whole = t0 + TT <= len && (t0 >= lo || t0 + TT <= a.sink) &&
                         __builtin_amdgcn_ballot_w64(vp < 0) == 0;
      if (!whole) {
#pragma unroll
        for (int e = 0; e < NM; ++e) {
          const int t = t0 + NM * g + e;
          // (no short circuits: selects, not branches)
          const bool on = (vp >= 0) & (t < len) & ((t >= lo) | (t < a.sink));
          z[e] = on ? z[e] : -INFINITY;
          val.keep(e, on);
        }
      }
      float m = z[0];
#pragma unroll
      for (int e = 1; e < NM; ++e) m = fmaxf(m, z[e]);
      m = fmaxf(m_run, over_groups_max(m) - M::kLower);
      const float ref = m == -INFINITY ? 0.f : m;
      const float sa = __builtin_amdgcn_exp2f(m_run - ref);      // (0 at the first tile)
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
      if (more) val.load(value_row(tn, vpn), a.tok_stride, n);
      i = in;
      t0 = tn;
      vp = vpn;
    }
    l_run = over_groups_sum(l_run);

    // The waves' parts meet in LDS.
    if (g == 0) {
      sm[wave][n] = m_run;
      sl[wave][n] = l_run;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) so[wave][n][M::channel(j, r, g)] = acc[j][r];
    __syncthreads();

    const RowShare share = row_share(start, rt.n, quota);
    const int parts = share.last - share.first + 1;
    // What a row ends as: outputs and log-sum-exp, or a partial for another join.
    auto finish = [&](int h, int c, float mm, float l, float o) {
      if (a.seg) {
        Partial* s = a.seg + q_row + h;
        s->o[c] = o;
        if (c == 0) {
          s->m = mm;
          s->l = l;
        }
        return;
      }
      a.out[(q_row + h) * kD + c] = l == 0.f ? 0.f : o / l;
      if (a.lse && c == 0) a.lse[q_row + h] = l == 0.f ? -INFINITY : (mm + log2f(l)) * kLn2;
    };
    float* slots = a.parts;
    for (int x = tid; x < heads * kD; x += kPagedThreads) {
      const int h = x / kD, c = x % kD;
      float mm = sm[0][h];
#pragma unroll
      for (int w = 1; w < kPagedWaves; ++w) mm = fmaxf(mm, sm[w][h]);
      float l = 0.f, o = 0.f;
#pragma unroll
      for (int w = 0; w < kPagedWaves; ++w) {
        const float f = sm[w][h] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm[w][h] - mm);
        l += sl[w][h] == 0.f ? 0.f : f * sl[w][h];
        o += f == 0.f ? 0.f : f * so[w][h][c];
      }
      if (parts == 1) {
        finish(h, c, mm, l, o);
      } else {
        float* slot = slots + (int64_t)part_slot(blockIdx.x, start, quota) * kPartFloats;
        st_dev(slot + 2 * kPagedHeads + h * kD + c, o);
        if (c == 0) {
          st_dev(slot + h, mm);
          st_dev(slot + kPagedHeads + h, l);
        }
      }
    }
    if (parts > 1) {
      unsigned* counter = a.counters + ((int64_t)seq * rows + row) * kRowStride;
      __builtin_amdgcn_s_waitcnt(0);               // this thread's stores are done
      __syncthreads();
      if (tid == 0)
        arrived = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __syncthreads();
      if (arrived == (unsigned)parts - 1u) {
        for (int x = tid; x < heads * kD; x += kPagedThreads) {
          const int h = x / kD, c = x % kD;
          float mm = -INFINITY, l = 0.f, o = 0.f;
          for (int w = share.first; w <= share.last; ++w) {
            const float* slot = slots + (int64_t)part_slot(w, start, quota) * kPartFloats;
            const float pm = ld_dev(slot + h), pl = ld_dev(slot + kPagedHeads + h);
            const float po = ld_dev(slot + 2 * kPagedHeads + h * kD + c);
            if (pl == 0.f) continue;               // no attended token there
            const float nm = fmaxf(mm, pm);
            const float ref = nm == -INFINITY ? 0.f : nm;
            const float fa = __builtin_amdgcn_exp2f(mm - ref), fb = __builtin_amdgcn_exp2f(pm - ref);
            l = l * fa + pl * fb;
            o = o * fa + po * fb;
            mm = nm;
          }
          finish(h, c, mm, l, o);
        }
        if (tid == 0) *counter = 0u;               // as the next call expects it
      }
    }
    start += rt.n;
    if (start >= end) break;
    __syncthreads();                               // LDS is read: the next row's parts go there
    if (++row == rows) {
      row = 0;
      ++seq;
      rt = tiles_of(seq);
    }
  }
}

size_t counters_bytes(int batch, int n_q_heads, int n_kv_heads) {
  const int hg = (n_q_heads / n_kv_heads + kPagedHeads - 1) / kPagedHeads;
  return round256((size_t)batch * n_kv_heads * hg * kRowStride * sizeof(unsigned));
}

}  // namespace

size_t paged_workspace_bytes(int batch, int n_q_heads, int n_kv_heads) {
  return counters_bytes(batch, n_q_heads, n_kv_heads) +
         2 * (size_t)kPagedGroups * kPartFloats * sizeof(float);
}

aatc_status launch_paged(PagedArgs a, aatc_dtype c_dtype, void* workspace, void* stream) {
  a.counters = static_cast<unsigned*>(workspace);
  a.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) +
                                     counters_bytes(a.batch, a.n_q_heads, a.n_kv_heads));
  const int tt = c_dtype == AATC_F32 ? Full32::kTokens : Half16<__bf16>::kTokens;
  const int64_t rows = (int64_t)a.batch * a.n_kv_heads * a.hg;
  const int64_t most = rows * std::max(1, (a.len_max + tt - 1) / tt);
  if (most > (1 << 30)) return AATC_E_UNSUPPORTED;
  const int grid = (int)std::min<int64_t>(kPagedGroups, (most + kQuotaMin - 1) / kQuotaMin);
  const hipStream_t st = (hipStream_t)stream;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kPagedThreads), 0, st, a);
    return hipGetLastError() == hipSuccess ? AATC_OK : AATC_E_DEVICE;
  };
  const bool same = a.q_dtype == (int)c_dtype;
  switch (c_dtype) {
    case AATC_F32: return launch(paged_kernel<Full32, 1>);
    case AATC_BF16:
      return same ? launch(paged_kernel<Half16<__bf16>, 1>) : launch(paged_kernel<Half16<__bf16>, 3>);
    default:
      return same ? launch(paged_kernel<Half16<_Float16>, 1>) : launch(paged_kernel<Half16<_Float16>, 3>);
  }
}

}  // namespace aatc
