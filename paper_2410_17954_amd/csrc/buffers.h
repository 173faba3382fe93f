// Raw buffers, the lane exchange of weight streams and SwiGLU, shared by the
// expert kernels.
#pragma once

#include "common.h"

namespace moe {

// Raw buffer over `elems` 16-bit values at p.
typedef __amdgpu_buffer_rsrc_t rsrc_t;
__device__ __forceinline__ rsrc_t make_rsrc(const uint16_t* p, int64_t elems) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(p), 0, (int)(uint32_t)(elems * 2),
                                           0x00027000);
}

// 16 bytes per lane of a raw buffer, from byte offset voff (lane) + soff (wave);
// past its end: zeros. NT: non-temporal.
template <bool NT>
__device__ __forceinline__ u32x4_t buf_load16(rsrc_t rs, uint32_t voff, uint32_t soff) {
  return __builtin_amdgcn_raw_buffer_load_b128(rs, (int)voff, (int)soff, NT ? 2 : 0);
}

__device__ __forceinline__ uint32_t ror8_into(uint32_t keep, uint32_t from, bool high) {
  // lanes 8..15 (high) or 0..7 of each row of 16 take `from` of the lane 8 away
  return high ? (uint32_t)__builtin_amdgcn_update_dpp((int)keep, (int)from, 0x128, 0xf, 0xc, false)
              : (uint32_t)__builtin_amdgcn_update_dpp((int)keep, (int)from, 0x128, 0xf, 0x3, false);
}

// silu(g) * u with the hardware exp2 and reciprocal (about 2 ulp of float32,
// far below the bf16 rounding of the result); exp2 overflows to +inf for very
// negative g, giving g * 0 * u = -0 as the exact expression does.
__device__ __forceinline__ float swiglu(float g, float u) {
  const float e = __builtin_amdgcn_exp2f(-g * 1.4426950408889634f);
  return g * __builtin_amdgcn_rcpf(1.f + e) * u;
}

}  // namespace moe
