// A wave's tile of the attention over pages: 32 tokens (16 in float32) of one KV head against up to
// 16 queries, scores = K Q^T and then O^T += V^T P^T on the matrix cores (paged.hip says how the two
// fit together).  Device code of the kernels that read pages.
#pragma once

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <cfloat>

#include "aatc.h"
#include "paged.h"
#include "params.h"

namespace aatc {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// The maximum of a part that has attended tokens, all with scores of -infinity (a part without
// attended tokens has -infinity and the sum 0).  Its sum is not 0, so that a head without any finite
// score ends as the NaN that its softmax is; beside finite scores it has no weight.
constexpr float kLowest = -FLT_MAX;
constexpr int kRsrcWord3 = 0x00020000;            // raw buffer descriptor word 3 (gfx950)
constexpr int kCoherent = 16;                     // cache policy sc1: device-coherent access

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

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

// FAR: keys and values are loaded past the caches.  Pools that do not fit there have nothing to
// gain from them (4 x 131072 tokens, 8 KV heads: 317.5 us, 358 through the caches; 1 x 32768 27.7
// and 30.7), smaller ones may be found there again (1 x 4000 tokens 14.7 and 13.0).  The pool is what
// counts, whatever part of it the sequences have.
constexpr int64_t kFarBytes = (int64_t)128 << 20;
inline bool pools_far(const PagedArgs& a, aatc_dtype c_dtype) {
  const int64_t page_bytes = ((int64_t)1 << a.page_shift) * a.n_kv_heads * kD *
                             (c_dtype == AATC_F32 ? 4 : 2);
  return 2 * page_bytes > kFarBytes / a.n_pages;                 // (both pools)
}
template <bool FAR, class V>
__device__ inline V load16(const char* p) {
  if constexpr (FAR) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
  else return *reinterpret_cast<const V*>(p);
}

// The two products on 16-bit types.  A lane's place: n = lane % 16, g = lane / 16.
template <class T, bool FAR>
struct Half16 {
  static constexpr bool kF16 = sizeof(T) == 2 && __is_same(T, _Float16);
  typedef T Elem;
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
  // A tile in LDS: piece c (16 bytes) of a token's row lies in the place c ^ turn_of(row), so that
  // the rows that a part of a wave reads at one time are in different banks.  Register u (of eight) of a
  // lane's keys is at (key_place ^ 64 key_flip(u)) + key_offset(u).
  static constexpr int kRow = 256;
  static __device__ int turn_of(int row) { return (row & 3) << 1 | (row & 8); }
  static __device__ int key_place(int n, int g) {
    const int row = key_token(0, n);
    return row * kRow + 16 * (g ^ turn_of(row));
  }
  static constexpr int key_flip(int u) { return u % 4; }
  static constexpr int key_offset(int u) { return u / 4 * 4 * kRow; }
  // Values are read turned (ds_read_b64_tr_b16: of sixteen lanes, lane 4 e + q reads four channels of
  // token e, lane i gets channel i of the four tokens): product j has channels 16 j + 0 .. 15, its
  // tokens 8 g + 4 x + e at (value_place ^ 32 j) + 4 kRow x.
  static constexpr bool kReadsTurned = true;
  static __device__ int value_place(int n, int g) {
    const int row = 8 * g + (n >> 2);
    return row * kRow + 16 * ((n >> 1 & 1) ^ turn_of(row)) + 8 * (n & 1);
  }
  static __device__ int turned_channel(int j, int i, int g) { return 16 * j + 4 * g + i; }

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
          r[u][kk] = load16<FAR, v4u>(row0 + u * 4 * tok_stride + 64 * kk + 16 * g);
    }
  };
  struct Values {
    v4u r[8];
    __device__ void load(const char* row0, int64_t tok_stride, int n) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        r[e] = load16<FAR, v4u>(row0 + e * tok_stride + 16 * n);
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

  // The product for several groups of 16 queries: the values are turned once.
  struct Turned {
    v4u a[8];
  };
  static __device__ void turn(const Values& v, Turned& t) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int d = 0; d < 4; ++d)
        t.a[j][d] = __builtin_amdgcn_perm(v.r[2 * d + 1][j / 2], v.r[2 * d][j / 2],
                                          j & 1 ? 0x07060302u : 0x05040100u);
  }
  // Token e of the lane's counts as zeros unless it is in `on` (bit e).
  static __device__ void keep_turned(Turned& t, unsigned on) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const uint32_t mask = (on >> (2 * d) & 1u ? 0xffffu : 0u) | (on >> (2 * d + 1) & 1u ? 0xffff0000u : 0u);
#pragma unroll
      for (int j = 0; j < 8; ++j) t.a[j][d] &= mask;
    }
  }
  // Whether any of the lane's values may be not finite, and those as zeros.
  static __device__ bool any_bad(const Turned& t) {
    Values v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v.r[j] = t.a[j];
    return any_bad(v);
  }
  static __device__ bool bad16(uint32_t x) {
    const uint32_t up = kF16 ? 0x7c00u : 0x7f80u;
    return (x & up) == up;
  }
  static __device__ void drop_bad(Turned& t) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const uint32_t x = t.a[j][d];
        t.a[j][d] = (bad16(x) ? 0u : x & 0xffffu) | (bad16(x >> 16) ? 0u : x & 0xffff0000u);
      }
  }
  // P as terms of 8 tokens.  bf16: the upper half of the number, the upper half of the rest, the rest
  // (exact: 8 bits each of 24).  f16: towards zero, then the rest to the nearest (2^-22 of it).
  struct Weights {
    v4u t[kTerms];
  };
  static __device__ Weights split(const float (&p)[kMine]) {
    Weights w;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      float x = p[2 * d], y = p[2 * d + 1];
      if constexpr (kF16) {
        const auto top = __builtin_amdgcn_cvt_pkrtz(x, y);
        typedef _Float16 v2h __attribute__((ext_vector_type(2)));
        float a, b;                                // x - top[0], y - top[1] (exact)
        asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(a) : "v"(top), "v"(x));
        asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(b) : "v"(top), "v"(y));
        const v2h rest = {(_Float16)a, (_Float16)b};
        w.t[0][d] = __builtin_bit_cast(uint32_t, top);
        w.t[1][d] = __builtin_bit_cast(uint32_t, rest);
      } else {
#pragma unroll
        for (int i = 0; i < kTerms; ++i) {
          w.t[i][d] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
          x -= __uint_as_float(__float_as_uint(x) & 0xffff0000u);
          y -= __uint_as_float(__float_as_uint(y) & 0xffff0000u);
        }
      }
    }
    return w;
  }
  static __device__ v4f add(const Turned& v, int j, const Weights& w, v4f acc) {
#pragma unroll
    for (int i = kTerms - 1; i >= 0; --i)
      acc = mfma(__builtin_bit_cast(v8, v.a[j]), __builtin_bit_cast(v8, w.t[i]), acc);
    return acc;
  }
  // Token e in the place of the first, if asked.
  static __device__ void take(Values& to, const Values& v, int e, bool on) {
#pragma unroll
    for (int i = 0; i < 4; ++i) to.r[0][i] = on ? v.r[e][i] : to.r[0][i];
  }
  // Whether any of the lane's values may be not finite (all bits of the exponent in some element).
  static __device__ bool any_bad(const Values& v) {
    typedef uint16_t v2 __attribute__((ext_vector_type(2)));
    const uint32_t up = kF16 ? 0x7c007c00u : 0x7f807f80u;
    v2 most = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int d = 0; d < 4; ++d)
        most = __builtin_elementwise_max(most, __builtin_bit_cast(v2, v.r[e][d] & up));
    return most[0] == (up & 0xffffu) || most[1] == (up & 0xffffu);
  }
  // Whether the lane's part of token e is not finite.
  static __device__ bool bad(const Values& v, int e) {
    const uint32_t up = kF16 ? 0x7c00u : 0x7f80u;
    bool b = false;
#pragma unroll
    for (int d = 0; d < 4; ++d)
      b |= ((v.r[e][d] & up) == up) | ((v.r[e][d] >> 16 & up) == up);
    return b;
  }
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
template <bool FAR>
struct Full32 {
  typedef float Elem;
  static constexpr int kTokens = 16;
  static constexpr int kMine = 4;                 // tokens 4 g .. 4 g + 3
  static constexpr float kLower = 0.f;
  static __device__ int key_token(int, int n) { return n; }
  static __device__ int key_block(int n) { return n >> 3; }
  static __device__ int value_block(int g) { return g >> 1; }
  // (as Half16's; values are read as rows: register u at (value_place ^ 16 value_flip(u)) +
  // value_offset(u))
  static constexpr int kRow = 512;
  static __device__ int turn_of(int row) { return row & 7; }
  static __device__ int key_place(int n, int g) { return n * kRow + 16 * (g ^ turn_of(n)); }
  static constexpr int key_flip(int u) { return u % 2; }
  static constexpr int key_offset(int u) { return u / 2 * 128; }
  static constexpr bool kReadsTurned = false;
  static __device__ int value_place(int n, int g) { return 4 * g * kRow + 16 * (n ^ turn_of(4 * g)); }
  static constexpr int value_flip(int u) { return u / 2; }
  static constexpr int value_offset(int u) { return u / 2 * kRow + u % 2 * 256; }
  static __device__ int turned_channel(int j, int i, int g) { return channel(j, i, g); }
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
      for (int c = 0; c < 8; ++c) r[c] = load16<FAR, v4f>(row0 + 64 * c + 16 * g);
    }
  };
  struct Values {
    v4f r[4][2];
    __device__ void load(const char* row0, int64_t tok_stride, int n) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < 2; ++c)
          r[e][c] = load16<FAR, v4f>(row0 + e * tok_stride + 256 * c + 16 * n);
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
  typedef Values Turned;
  static __device__ void turn(const Values& v, Turned& t) { t = v; }
  struct Weights {
    float p[kMine];
  };
  static __device__ Weights split(const float (&p)[kMine]) {
    Weights w;
#pragma unroll
    for (int e = 0; e < kMine; ++e) w.p[e] = p[e];
    return w;
  }
  static __device__ v4f add(const Turned& v, int j, const Weights& w, v4f acc) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) acc = mfma(v.r[i][j >> 2][j & 3], w.p[i], acc);
    return acc;
  }
  static __device__ void take(Values& to, const Values& v, int e, bool on) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) to.r[0][c][i] = on ? v.r[e][c][i] : to.r[0][c][i];
  }
  static __device__ bool any_bad(const Values& v) {
    float most = 0.f;                              // (x - x is not 0 for those alone)
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) most += v.r[e][c][i] - v.r[e][c][i];
    return !(most == 0.f);
  }
  static __device__ bool bad(const Values& v, int e) {
    bool b = false;
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) b |= !(fabsf(v.r[e][c][i]) < INFINITY);
    return b;
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

// What the weights of scores up to `top` (exponents of 2) are relative to: kLower below it, so that small
// ones stay off f16's denormals; the score itself where the difference, rounded to the places of large
// scores (from 2^25 on), would leave weights of 2^16, beyond f16.
template <class M>
__device__ inline float reference_of(float top) {
  const float low = top - M::kLower;
  return M::kLower > 0.f && top - low > 15.f ? top : low;
}

// tanh to a few ulps: for small |x| the first terms of its odd series (the next is 4e-8 of x at
// 0.55), else from exp(-2 |x|).
__device__ inline float tanh_of(float x) {
  const float y = fabsf(x), s = y * y;
  float r = 0.0014558343f;                         // 929569 / 638512875, 21844 / 6081075, ...
  r = fmaf(-r, s, 0.003592128f);
  r = fmaf(-r, s, 0.0088632356f);
  r = fmaf(-r, s, 0.021869488f);
  r = fmaf(-r, s, 0.053968254f);
  r = fmaf(-r, s, 0.13333334f);
  r = fmaf(-r, s, 0.33333334f);
  const float small = fmaf(-r * s, y, y);
  const float e = __builtin_amdgcn_exp2f(-2.f * kLog2e * y);
  const float large = (1.f - e) / (1.f + e);
  return copysignf(y < 0.55f ? small : large, x);
}

}  // namespace
}  // namespace aatc
