// The largest and the sum of a number of every lane, in six steps of data-parallel primitives; the same in all lanes.  All
// lanes have to be on: one that is off has nothing to give.
#pragma once
#include <hip/hip_runtime.h>

namespace mip {

// x of the lane that CTRL names; `other` where there is none, or where ROWS leaves a row of 16 lanes out.
template <int CTRL, int ROWS>
__device__ __forceinline__ float moved(float x, float other) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(other), __float_as_int(x), CTRL, ROWS, 0xf, false));
}
constexpr int SHR_1 = 0x111, SHR_2 = 0x112, SHR_4 = 0x114, SHR_8 = 0x118, BROADCAST_15 = 0x142, BROADCAST_31 = 0x143;

__device__ __forceinline__ float last_lane(float x) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63)); }
__device__ __forceinline__ float wave_most(float v) {
  v = __builtin_fmaxf(v, moved<SHR_1, 0xf>(v, v));
  v = __builtin_fmaxf(v, moved<SHR_2, 0xf>(v, v));
  v = __builtin_fmaxf(v, moved<SHR_4, 0xf>(v, v));
  v = __builtin_fmaxf(v, moved<SHR_8, 0xf>(v, v));
  v = __builtin_fmaxf(v, moved<BROADCAST_15, 0xa>(v, v));
  v = __builtin_fmaxf(v, moved<BROADCAST_31, 0xc>(v, v));
  return last_lane(v);
}
__device__ __forceinline__ float wave_sum(float v) {
  v += moved<SHR_1, 0xf>(v, 0.0f);
  v += moved<SHR_2, 0xf>(v, 0.0f);
  v += moved<SHR_4, 0xf>(v, 0.0f);
  v += moved<SHR_8, 0xf>(v, 0.0f);
  v += moved<BROADCAST_15, 0xa>(v, 0.0f);
  v += moved<BROADCAST_31, 0xc>(v, 0.0f);
  return last_lane(v);
}

}  // namespace mip
