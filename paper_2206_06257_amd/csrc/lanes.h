// Exchanges between the lanes of a wavefront.
#pragma once
#include "common.h"

namespace dat {

// Reductions over L = 16 or 64 neighbouring lanes by DPP (a vector instruction a step, no LDS); every lane has the result.
template <int CTRL, int ROWS> __device__ __forceinline__ int dpp(int v) { return __builtin_amdgcn_update_dpp(v, v, CTRL, ROWS, 0xf, false); }
template <int L, typename F> __device__ __forceinline__ int lanes_reduce(int v, F f) {
  v = f(v, dpp<0xb1, 0xf>(v));                   // the other of two, of two pairs, of half a row, of a row of 16
  v = f(v, dpp<0x4e, 0xf>(v));
  if (L >= 16) v = f(v, dpp<0x141, 0xf>(v));
  if (L >= 16) v = f(v, dpp<0x140, 0xf>(v));
  if (L == 64) {
    const int a = __builtin_amdgcn_readlane(v, 15), b = __builtin_amdgcn_readlane(v, 31), c = __builtin_amdgcn_readlane(v, 47),
              d = __builtin_amdgcn_readlane(v, 63);
    v = f(f(a, b), f(c, d));
  }
  return v;
}
__device__ __forceinline__ float maximum(float a, float b) { return __builtin_elementwise_maximum(a, b); }   // a NaN stays
template <int L> __device__ __forceinline__ float lanes_max(float v) {
  return __int_as_float(lanes_reduce<L>(__float_as_int(v), [](int a, int b) { return __float_as_int(maximum(__int_as_float(a), __int_as_float(b))); }));
}
template <int L> __device__ __forceinline__ float lanes_sum(float v) {
  return __int_as_float(lanes_reduce<L>(__float_as_int(v), [](int a, int b) { return __float_as_int(__int_as_float(a) + __int_as_float(b)); }));
}
template <int L> __device__ __forceinline__ int lanes_min(int v) { return lanes_reduce<L>(v, [](int a, int b) { return min(a, b); }); }

}  // namespace dat
