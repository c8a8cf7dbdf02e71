// Scans over the lanes of a wave.  Device code; all lanes active.
#pragma once

#include <hip/hip_runtime.h>

namespace aatc {
namespace {

// Over a wave, by shifts within rows of 16 lanes and broadcasts of rows' last lanes: lane l gets f of the
// lanes up to l (the last one f of all).  `none`: what f leaves as it is.
template <class F>
__device__ inline int wave_scan(int x, int none, F f) {
  x = f(x, __builtin_amdgcn_update_dpp(none, x, 0x111, 0xf, 0xf, false));      // row_shr:1
  x = f(x, __builtin_amdgcn_update_dpp(none, x, 0x112, 0xf, 0xf, false));
  x = f(x, __builtin_amdgcn_update_dpp(none, x, 0x114, 0xf, 0xf, false));
  x = f(x, __builtin_amdgcn_update_dpp(none, x, 0x118, 0xf, 0xf, false));
  x = f(x, __builtin_amdgcn_update_dpp(none, x, 0x142, 0xa, 0xf, false));      // row_bcast:15
  x = f(x, __builtin_amdgcn_update_dpp(none, x, 0x143, 0xc, 0xf, false));      // row_bcast:31
  return x;
}
__device__ inline int wave_scan_sum(int x) {
  return wave_scan(x, 0, [](int a, int b) { return a + b; });
}
__device__ inline int wave_total(int x) { return __builtin_amdgcn_readlane(wave_scan_sum(x), 63); }

// Over each row of 16 lanes, by rotations: every lane gets the row's largest.
template <int CTRL>
__device__ inline float row_max_step(float x) {
  return fmaxf(x, __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf,
                                                                         0xf, true)));
}
__device__ inline float row_max(float x) {
  return row_max_step<0x121>(row_max_step<0x122>(row_max_step<0x124>(row_max_step<0x128>(x))));
}

}  // namespace
}  // namespace aatc
