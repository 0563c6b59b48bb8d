// Device helpers of the operators of seedq_mx4.h.
#pragma once

#include <algorithm>

#include "seedq_mx4_internal.h"
#include "seedq_ops_device.h"

namespace seedq {

// 2^(e - 127) as the conversions take it.
__device__ __forceinline__ float mx_scale(uint32_t e) { return __builtin_bit_cast(float, e << 23); }

__device__ __forceinline__ void store_y(void* y, int ytype, int64_t at, float v) {
  if (ytype == SEEDQ_F32) static_cast<float*>(y)[at] = v;
  else static_cast<uint16_t*>(y)[at] = ytype == SEEDQ_F16 ? F16::narrow(v) : BF16::narrow(v);
}

// 16 bytes a lane to LDS, lane after lane.
__device__ __forceinline__ void to_lds16(const void* from, void* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from),
                                   (__attribute__((address_space(3))) void*)(to), 16, 0, 0);
}

// 16 bytes anywhere.
typedef uint32x4 uint32x4_byte __attribute__((aligned(1)));

// 16 bytes without their first n (none where n < 0), zeros after the last; n is the same
// for all lanes.
__device__ __forceinline__ uint32x4 after_bytes(uint32x4 v, int64_t n) {
  if (n <= 0) return v;
  const int m = int(std::min<int64_t>(n, 16));
  if (m & 16) return uint32x4{0u, 0u, 0u, 0u};
  if (m & 8) v = uint32x4{v[2], v[3], 0u, 0u};
  if (m & 4) v = uint32x4{v[1], v[2], v[3], 0u};
  if (m & 3)
    v = uint32x4{__builtin_amdgcn_alignbyte(v[1], v[0], m & 3), __builtin_amdgcn_alignbyte(v[2], v[1], m & 3),
                 __builtin_amdgcn_alignbyte(v[3], v[2], m & 3), v[3] >> (8 * (m & 3))};
  return v;
}

}  // namespace seedq
