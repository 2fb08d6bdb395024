// Reductions and prefixes over the lanes of a wave by data-parallel moves, which
// cost an instruction where a shuffle goes through the LDS.  After the six steps of a
// reduction (or inclusive prefix: 1, 2, 4 and 8 lanes down within a row of sixteen,
// then a row's last lane to the next row, lane 31 to the upper half) the last lane
// has the whole.  All lanes of the wave take part.
#pragma once

#include "device_util.h"

namespace spade {

template <int STEP>
__device__ __forceinline__ uint32_t prefix_step(uint32_t v, uint32_t none) {
  constexpr int ctrl = STEP < 4 ? 0x110 + (1 << STEP) : STEP == 4 ? 0x142 : 0x143;
  constexpr int rows = STEP < 4 ? 0xf : STEP == 4 ? 0xa : 0xc;
  return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, ctrl, rows, 0xf, false);
}
template <int STEP>
__device__ __forceinline__ uint64_t prefix_step(uint64_t v, uint64_t none) {
  return (uint64_t)prefix_step<STEP>((uint32_t)(v >> 32), (uint32_t)(none >> 32)) << 32 |
         prefix_step<STEP>((uint32_t)v, (uint32_t)none);
}
template <int STEP>
__device__ __forceinline__ double prefix_step(double v, double none) {
  return __longlong_as_double(
      (long long)prefix_step<STEP>((uint64_t)__double_as_longlong(v), (uint64_t)__double_as_longlong(none)));
}
template <int STEP>
__device__ __forceinline__ float prefix_step(float v, float none) {
  return __uint_as_float(prefix_step<STEP>(__float_as_uint(v), __float_as_uint(none)));
}
template <int STEP>
__device__ __forceinline__ int prefix_step(int v, int none) {
  return (int)prefix_step<STEP>((uint32_t)v, (uint32_t)none);
}

// v of lane l, the same for all
__device__ __forceinline__ uint32_t from_lane(uint32_t v, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); }
__device__ __forceinline__ int from_lane(int v, int l) { return __builtin_amdgcn_readlane(v, l); }
__device__ __forceinline__ float from_lane(float v, int l) { return __uint_as_float(from_lane(__float_as_uint(v), l)); }
__device__ __forceinline__ uint64_t from_lane(uint64_t v, int l) {
  return (uint64_t)from_lane((uint32_t)(v >> 32), l) << 32 | from_lane((uint32_t)v, l);
}
__device__ __forceinline__ double from_lane(double v, int l) {
  return __longlong_as_double((long long)from_lane((uint64_t)__double_as_longlong(v), l));
}

// f over all lanes (f(x, x) = x), in the last
template <typename T, typename F>
__device__ __forceinline__ T all_lanes(T v, F f) {
  v = f(v, prefix_step<0>(v, v));
  v = f(v, prefix_step<1>(v, v));
  v = f(v, prefix_step<2>(v, v));
  v = f(v, prefix_step<3>(v, v));
  v = f(v, prefix_step<4>(v, v));
  return f(v, prefix_step<5>(v, v));
}
// inclusive prefix sums
template <typename T>
__device__ __forceinline__ T prefix_sum(T v) {
  v += prefix_step<0>(v, (T)0);
  v += prefix_step<1>(v, (T)0);
  v += prefix_step<2>(v, (T)0);
  v += prefix_step<3>(v, (T)0);
  v += prefix_step<4>(v, (T)0);
  return v + prefix_step<5>(v, (T)0);
}

}  // namespace spade
