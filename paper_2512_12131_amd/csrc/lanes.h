// Sums and maxima over a wavefront's lanes by DPP moves, which stay in the vector unit (a __shfl goes through the LDS crossbar: for the plan of a
// fork, 2 prefix sums, 5.5 us that way and 4.8 so).
#pragma once
#include "common.h"

namespace lrb {
namespace {

// v of the lane that a DPP control names, `none` where there is none
template <int CTRL, int ROWS>
__device__ __forceinline__ int from_lane(int v, int none) { return __builtin_amdgcn_update_dpp(none, v, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t from_lane(uint32_t v, uint32_t none) { return (uint32_t)from_lane<CTRL, ROWS>((int)v, (int)none); }
template <int CTRL, int ROWS>
__device__ __forceinline__ float from_lane(float v, float none) { return __int_as_float(from_lane<CTRL, ROWS>(__float_as_int(v), __float_as_int(none))); }
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t from_lane(int64_t v, int64_t none) {
  return (int64_t)((uint64_t)(uint32_t)from_lane<CTRL, ROWS>((int)(v >> 32), (int)(none >> 32)) << 32 | (uint32_t)from_lane<CTRL, ROWS>((int)v, (int)none));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double from_lane(double v, double none) {
  return __longlong_as_double(from_lane<CTRL, ROWS>((int64_t)__double_as_longlong(v), (int64_t)__double_as_longlong(none)));
}
__device__ __forceinline__ uint32_t value_of_lane(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ float value_of_lane(float v, int lane) { return __uint_as_float(value_of_lane(__float_as_uint(v), lane)); }
__device__ __forceinline__ double value_of_lane(double v, int lane) {
  return __hiloint2double((int)value_of_lane((uint32_t)__double2hiint(v), lane), (int)value_of_lane((uint32_t)__double2loint(v), lane));
}

// f over the lanes up to this one, where `none` changes nothing
template <class V, class F>
__device__ __forceinline__ V wave_scan(V v, V none, F f) {
  v = f(v, from_lane<0x111, 0xf>(v, none));      // row_shr:1, 2, 4, 8: within 16 lanes
  v = f(v, from_lane<0x112, 0xf>(v, none));
  v = f(v, from_lane<0x114, 0xf>(v, none));
  v = f(v, from_lane<0x118, 0xf>(v, none));
  v = f(v, from_lane<0x142, 0xa>(v, none));      // row_bcast:15 into the second and fourth 16
  return f(v, from_lane<0x143, 0xc>(v, none));   // row_bcast:31 into the upper 32
}
template <class V>
__device__ __forceinline__ V wave_prefix(V v) {
  return wave_scan(v, V(0), [](V a, V b) { return a + b; });
}
// over all lanes, the same in all of them
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  return value_of_lane(wave_scan(v, 0u, [](uint32_t a, uint32_t b) { return max(a, b); }), 63);
}
__device__ __forceinline__ float wave_max(float v) {
  return value_of_lane(wave_scan(v, -INFINITY, [](float a, float b) { return fmaxf(a, b); }), 63);
}
__device__ __forceinline__ double wave_sum(double v) { return value_of_lane(wave_prefix(v), 63); }
// over 16 lanes next to each other, the same in all of them
template <class V, class F>
__device__ __forceinline__ V row_all(V v, F f) {
  v = f(v, from_lane<0x128, 0xf>(v, v));         // row_ror:8, 4, 2, 1
  v = f(v, from_lane<0x124, 0xf>(v, v));
  v = f(v, from_lane<0x122, 0xf>(v, v));
  return f(v, from_lane<0x121, 0xf>(v, v));
}

}  // namespace
}  // namespace lrb
