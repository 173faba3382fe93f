// Reductions over rows of 16 lanes (gfx950 DPP moves).
#pragma once

#include "common.h"

namespace moe {

// ---------------------------------------------------------------- rows of 16
// Every reduction of the decision runs over a row of 16 lanes (one token per
// row, four per wave) with DPP moves: quad_perm [1,0,3,2], quad_perm
// [2,3,0,1], row_half_mirror, row_mirror. After the four steps every lane of
// the row holds the row's result.
constexpr int kRowLanes = 16;

template <int CTRL>
__device__ __forceinline__ int dpp_i32(int v) {
  return __builtin_amdgcn_mov_dpp(v, CTRL, 0xF, 0xF, true);
}
template <int CTRL>
__device__ __forceinline__ int dpp(int v) { return dpp_i32<CTRL>(v); }
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(dpp_i32<CTRL>(__float_as_int(v)));
}
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
  const uint64_t b = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = (uint32_t)dpp_i32<CTRL>((int)(uint32_t)b);
  const uint32_t hi = (uint32_t)dpp_i32<CTRL>((int)(uint32_t)(b >> 32));
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}

// Arg-max under the order (larger value first, then lower index); e < 0
// marks an empty slot.
template <int C, typename VT>
__device__ __forceinline__ void argmax_step(VT& v, int& e) {
  const VT ov = dpp<C>(v);
  const int oe = dpp<C>(e);
  if (oe >= 0 && (e < 0 || ov > v || (ov == v && oe < e))) {
    v = ov;
    e = oe;
  }
}
template <typename VT>
__device__ __forceinline__ void row_argmax(VT& v, int& e) {
  argmax_step<0xB1>(v, e);
  argmax_step<0x4E>(v, e);
  argmax_step<0x141>(v, e);
  argmax_step<0x140>(v, e);
}

}  // namespace moe
