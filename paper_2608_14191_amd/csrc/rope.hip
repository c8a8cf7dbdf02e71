// Rotary positions, alone and on the way into the pages of a cache.
//
// Pair i of a head (channels (i, i + half) or (2 i, 2 i + 1)) at position p is turned by the
// angle p f_i and scaled:  (a, b) -> factor (a cos - b sin, b cos + a sin);  sign = -1 turns
// back (the adjoint: the gradient of the forward rotation).  The angle is taken in 64 bits, as
// revolutions p f_i / 2 pi less the nearest whole number, so that far positions lose nothing;
// sine and cosine of what is left, the products and their sum are in 32 bits, rounded once to
// the output's type.
//
// Bound by memory: 16-byte loads and stores, a wave to a token and some of its heads, whose
// sines it computes once (a lane each) while its loads are on their way.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "paged.h"
#include "params.h"

namespace aatc {
namespace {

constexpr int kTurnThreads = 256;
constexpr int kTurnWaves = kTurnThreads / 64;
constexpr int64_t kFarBytes = (int64_t)128 << 20;

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

template <int DT>
struct Elem;
template <>
struct Elem<AATC_F32> {
  using type = float;
  static __device__ float get(float x) { return x; }
  static __device__ float put(float x) { return x; }
};
template <>
struct Elem<AATC_BF16> {
  using type = __bf16;
  static __device__ float get(__bf16 x) { return (float)x; }
  static __device__ __bf16 put(float x) { return (__bf16)x; }
};
template <>
struct Elem<AATC_F16> {
  using type = _Float16;
  static __device__ float get(_Float16 x) { return (float)x; }
  // (The compiler may not see where x comes from: a product and sum that it rounds to f16 in one
  // instruction, in some instances of the kernel only, would differ from the float32 sum's rounding.)
  static __device__ _Float16 put(float x) {
    asm("" : "+v"(x));
    return (_Float16)x;
  }
};

// The turned pair.  The same operations in every instance of the kernel, so that a token's bits do
// not depend on its row's alignment or on how many others the call has.
__device__ inline float turned_low(float a, float b, float2 w) { return fmaf(a, w.x, -(b * w.y)); }
__device__ inline float turned_high(float a, float b, float2 w) { return fmaf(a, w.y, b * w.x); }

template <class T, int E>
struct alignas(sizeof(T) * E < 16 ? sizeof(T) * E : 16) Chunk {
  T e[E];
};

// FAR: past the caches (tokens that would not stay in them: 65536 of eight float32 heads
// 98.7 us, 104.4 through the caches; 4096 tokens of 32 bf16 heads 15.5, 12.7 through them).
template <bool FAR, class C>
__device__ inline void put_chunk(void* p, const C& c) {
  if constexpr (FAR && sizeof(C) == 16)
    __builtin_nontemporal_store(__builtin_bit_cast(v4u, c), static_cast<v4u*>(p));
  else
    *static_cast<C*>(p) = c;
}

template <bool FAR, class C>
__device__ inline C get_chunk(const void* p) {
  if constexpr (FAR && sizeof(C) == 16)
    return __builtin_bit_cast(C, __builtin_nontemporal_load(static_cast<const v4u*>(p)));
  else
    return *static_cast<const C*>(p);
}

// LDS written by other lanes of the wave: its accesses are in order, the compiler keeps them so.
__device__ inline void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// How a head's row is moved.  Whole: in 16-byte chunks, with a lane's partners in a chunk of its own
// (rows 16-byte aligned, and half a multiple of a chunk's elements unless pairs are interleaved).
// Shuffled: in chunks, the partners by way of LDS (half of any size: 32534 tokens of eight bf16
// heads, 2 channels rotated, 75.0 us channel by channel, 39.2 so).  Single: channel by channel
// (rows of any alignment).
enum Path { kWhole, kShuffled, kSingle };

// XD: type of the tokens and of q_out, CD: of the pages; INTER: interleaved pairs.
template <int XD, int CD, bool INTER, Path PATH, bool FAR>
__global__ __launch_bounds__(kTurnThreads) void turn_kernel(TurnArgs a, int heads_per_wave) {
  using X = Elem<XD>;
  using C = Elem<CD>;
  using XT = typename X::type;
  using CT = typename C::type;
  __shared__ float2 cs[kTurnWaves][kD / 2];
  __shared__ __align__(16) XT mix[kTurnWaves][PATH == kShuffled ? 64 * 16 / sizeof(XT) : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t tok = a.tok0 + (int64_t)blockIdx.x * kTurnWaves + wave;
  const bool in = tok < a.n_tok;
  const int p = in ? a.pos[tok] : 0;
  const bool on = in && !(a.skip_negative && p < 0);
  if (on && lane < a.half) {
    const double rev = (double)p * a.freq[lane] * 0.15915494309189533577;   // 1 / 2 pi
    float s, c;
    sincospif((float)(2.0 * (rev - rint(rev))), &s, &c);
    cs[wave][lane] = make_float2(a.factor * c, a.sign * a.factor * s);
  }
  __syncthreads();
  if (!on) return;
  // The token's slot in the pages (-1: none).
  int64_t slot = -1;
  if (a.heads[1] > 0) {
    const int64_t row = a.seq ? a.seq[tok] : tok;
    const int at = p >> a.page_shift;
    if (row >= 0 && row < a.rows && at < a.max_pages) {
      const int page = a.table[row * a.table_stride + at];
      if (page >= 0 && page < a.n_pages)
        slot = page * a.page_stride + (p & ((1 << a.page_shift) - 1)) * a.tok_stride;
    }
  }
  const int half = a.half, rot = 2 * half;
  const int turned = a.heads[0] + a.heads[1], all = turned + a.heads[2];
  const int h_end = min(all, (int)(blockIdx.y + 1) * heads_per_wave);
  // Source of head h and where it goes: q_out, or a page (null: nowhere).
  auto source = [&](int h) -> const XT* {
    const int part = h < a.heads[0] ? 0 : h < turned ? 1 : 2;
    const int hh = h - (part == 0 ? 0 : part == 1 ? a.heads[0] : turned);
    return static_cast<const XT*>(a.x[part]) + tok * a.x_stride[part] + hh * kD;
  };
  auto q_dest = [&](int h) { return static_cast<XT*>(a.q_out) + tok * a.q_out_stride + h * kD; };
  auto page_dest = [&](int h) {
    const int hh = h - (h < turned ? a.heads[0] : turned);
    return static_cast<CT*>(h < turned ? a.k_pages : a.v_pages) + slot + hh * a.head_stride;
  };
  constexpr int E = 16 / sizeof(XT);                   // elements of a chunk
  if constexpr (PATH == kWhole) {
    using XC = Chunk<XT, E>;
    using CC = Chunk<CT, E>;
    // Lanes of a head: two chunks each, E apart in the head by 128 / 2, or by `half` for the
    // pairs of the half layout.
    constexpr int LH = kD / (2 * E), HW = 64 / LH;     // lanes per head, heads at a time
    const int sub = lane % LH;
    for (int h = blockIdx.y * heads_per_wave + lane / LH; h < h_end; h += HW) {
      const bool to_q = h < a.heads[0], turn = h < turned;
      if (!to_q && slot < 0) continue;
      const XT* src = source(h);
      XT* dq = to_q ? q_dest(h) : nullptr;
      CT* dc = to_q ? nullptr : page_dest(h);
      auto store = [&](int c, const float (&y)[E]) {
        if (to_q) {
          XC o;
#pragma unroll
          for (int e = 0; e < E; ++e) o.e[e] = X::put(y[e]);
          put_chunk<FAR>(dq + c, o);
        } else {
          CC o;
#pragma unroll
          for (int e = 0; e < E; ++e) o.e[e] = C::put(y[e]);
          put_chunk<FAR>(dc + c, o);
        }
      };
      auto pass = [&](int c) {                         // a chunk that is not turned
        const XC x = get_chunk<FAR, XC>(src + c);
        if (to_q) {
          if (a.copy_rest) put_chunk<FAR>(dq + c, x);
          return;
        }
        float y[E];
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = X::get(x.e[e]);
        store(c, y);
      };
      if (!turn) {
        pass(E * sub);
        pass(E * (sub + LH));
      } else if constexpr (INTER) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int c = E * (sub + LH * u);
          if (c >= rot) {
            pass(c);
            continue;
          }
          const XC x = get_chunk<FAR, XC>(src + c);
          float y[E];
#pragma unroll
          for (int e = 0; e < E; e += 2) {
            const int i = (c + e) / 2;
            const float2 w = cs[wave][i < half ? i : 0];
            const float u0 = X::get(x.e[e]), u1 = X::get(x.e[e + 1]);
            y[e] = i < half ? turned_low(u0, u1, w) : u0;
            y[e + 1] = i < half ? turned_high(u0, u1, w) : u1;
          }
          store(c, y);
        }
      } else {
        if (E * sub < half) {
          const int c = E * sub;
          const XC x0 = get_chunk<FAR, XC>(src + c);
          const XC x1 = get_chunk<FAR, XC>(src + half + c);
          float y0[E], y1[E];
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float2 w = cs[wave][c + e];
            const float u0 = X::get(x0.e[e]), u1 = X::get(x1.e[e]);
            y0[e] = turned_low(u0, u1, w);
            y1[e] = turned_high(u0, u1, w);
          }
          store(c, y0);
          store(half + c, y1);
        }
        for (int c = rot + E * sub; c < kD; c += E * LH) pass(c);
      }
    }
  } else if constexpr (PATH == kShuffled) {
    using XC = Chunk<XT, E>;
    using CC = Chunk<CT, E>;
    constexpr int LH = kD / E, HW = 64 / LH;           // lanes per head, heads at a time
    const int c = E * (lane % LH);
    XT* row = mix[wave] + lane / LH * kD;
    for (int h = blockIdx.y * heads_per_wave + lane / LH; h < h_end; h += HW) {
      const bool to_q = h < a.heads[0], turn = h < turned;
      if (!to_q && slot < 0) continue;
      const XC x = get_chunk<FAR, XC>(source(h) + c);
      if (turn) *reinterpret_cast<XC*>(row + c) = x;
      wave_sync();
      float y[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        y[e] = X::get(x.e[e]);
        const int i = c + e;
        if (turn && i < rot) {
          const bool low = i < half;
          const float2 w = cs[wave][low ? i : i - half];
          const float other = X::get(row[low ? i + half : i - half]);
          y[e] = low ? turned_low(y[e], other, w) : turned_high(other, y[e], w);
        }
      }
      wave_sync();
      if (to_q) {
        XC o = x;                                      // (channels behind rot keep their bits)
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (c + e < rot) o.e[e] = X::put(y[e]);
        if (c < rot || a.copy_rest) put_chunk<FAR>(q_dest(h) + c, o);
      } else {
        CC o;
#pragma unroll
        for (int e = 0; e < E; ++e) o.e[e] = C::put(y[e]);
        put_chunk<FAR>(page_dest(h) + c, o);
      }
    }
  } else {
    for (int h = blockIdx.y * heads_per_wave; h < h_end; ++h) {
      const bool to_q = h < a.heads[0], turn = h < turned;
      if (!to_q && slot < 0) continue;
      const XT* src = source(h);
      XT* dq = to_q ? q_dest(h) : nullptr;
      CT* dc = to_q ? nullptr : page_dest(h);
      auto put = [&](int c, float y) {
        if (to_q) dq[c] = X::put(y);
        else dc[c] = C::put(y);
      };
      if (turn && lane < half) {
        const int c0 = INTER ? 2 * lane : lane, c1 = INTER ? 2 * lane + 1 : lane + half;
        const float2 w = cs[wave][lane];
        const float u0 = X::get(src[c0]), u1 = X::get(src[c1]);
        put(c0, turned_low(u0, u1, w));
        put(c1, turned_high(u0, u1, w));
      }
      for (int c = (turn ? rot : 0) + lane; c < kD; c += 64) {
        if (!to_q) put(c, X::get(src[c]));
        else if (a.copy_rest) dq[c] = src[c];
      }
    }
  }
}

template <int XD, int CD>
aatc_status launch_turn_types(TurnArgs a, int layout, Path path, hipStream_t st) {
  // (A launch has less than 2^32 threads.)
  constexpr int64_t kMost = (int64_t)1 << 25;
  for (; a.n_tok - a.tok0 > kMost; a.tok0 += kMost) {
    TurnArgs piece = a;
    piece.n_tok = a.tok0 + kMost;
    const aatc_status e = launch_turn_types<XD, CD>(piece, layout, path, st);
    if (e != AATC_OK) return e;
  }
  const int all = a.heads[0] + a.heads[1] + a.heads[2];
  const int64_t blocks = (a.n_tok - a.tok0 + kTurnWaves - 1) / kTurnWaves;
  // A wave takes up to 32 heads of its token; with few tokens fewer, so that the chip's compute
  // units all have some.
  int per = all < 32 ? all : 32;
  while (per > 8 && blocks * ((all + per - 1) / per) < 512) per = (per + 1) / 2;
  const dim3 grid((unsigned)blocks, (unsigned)((all + per - 1) / per));
  const bool inter = layout == AATC_ROPE_INTERLEAVED;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kTurnThreads), 0, st, a, per);
  };
  const bool far = a.n_tok * all * kD * (int64_t)sizeof(typename Elem<XD>::type) > kFarBytes;
  if (path == kSingle)
    inter ? launch(turn_kernel<XD, CD, true, kSingle, false>)
          : launch(turn_kernel<XD, CD, false, kSingle, false>);
  else if (path == kShuffled)
    launch(turn_kernel<XD, CD, false, kShuffled, false>);
  else if (far)
    inter ? launch(turn_kernel<XD, CD, true, kWhole, true>)
          : launch(turn_kernel<XD, CD, false, kWhole, true>);
  else
    inter ? launch(turn_kernel<XD, CD, true, kWhole, false>)
          : launch(turn_kernel<XD, CD, false, kWhole, false>);
  return hipGetLastError() == hipSuccess ? AATC_OK : AATC_E_DEVICE;
}

template <int XD>
aatc_status launch_turn_x(const TurnArgs& a, aatc_dtype c, int layout, Path path, hipStream_t st) {
  switch (c) {
    case AATC_F32: return launch_turn_types<XD, AATC_F32>(a, layout, path, st);
    case AATC_BF16: return launch_turn_types<XD, AATC_BF16>(a, layout, path, st);
    default: return launch_turn_types<XD, AATC_F16>(a, layout, path, st);
  }
}

}  // namespace

aatc_status launch_turn(const TurnArgs& a, aatc_dtype x_dtype, aatc_dtype c_dtype, int layout,
                        void* stream) {
  const int size = x_dtype == AATC_F32 ? 4 : 2, e = 16 / size;
  bool even = true;                                    // rows of 16-byte chunks
  for (int i = 0; i < 3; ++i)
    if (a.heads[i] > 0)
      even = even && reinterpret_cast<uintptr_t>(a.x[i]) % 16 == 0 && a.x_stride[i] % e == 0;
  if (a.heads[0] > 0)
    even = even && reinterpret_cast<uintptr_t>(a.q_out) % 16 == 0 && a.q_out_stride % e == 0;
  const bool pairs = layout == AATC_ROPE_INTERLEAVED || a.half % e == 0;
  const Path path = !even ? kSingle : pairs ? kWhole : kShuffled;
  const hipStream_t st = (hipStream_t)stream;
  switch (x_dtype) {
    case AATC_F32: return launch_turn_x<AATC_F32>(a, c_dtype, layout, path, st);
    case AATC_BF16: return launch_turn_x<AATC_BF16>(a, c_dtype, layout, path, st);
    default: return launch_turn_x<AATC_F16>(a, c_dtype, layout, path, st);
  }
}

}  // namespace aatc
