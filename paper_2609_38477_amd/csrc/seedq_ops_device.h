// Device helpers of the operators of seedq_ops.h: element types and their loads.
#pragma once

#include "seedq_ops_internal.h"

namespace seedq {

struct F32 {
  using raw = float;
  __device__ static __forceinline__ float widen(raw v) { return v; }
  __device__ static __forceinline__ raw narrow(float v) { return v; }
};
struct F16 {
  using raw = uint16_t;
  __device__ static __forceinline__ float widen(raw v) {
    return float(__builtin_bit_cast(_Float16, v));
  }
  __device__ static __forceinline__ raw narrow(float v) {   // to nearest even
    return __builtin_bit_cast(uint16_t, _Float16(v));
  }
};
struct BF16 {
  using raw = uint16_t;
  __device__ static __forceinline__ float widen(raw v) {
    return __builtin_bit_cast(float, uint32_t(v) << 16);
  }
  __device__ static __forceinline__ raw narrow(float v) {   // to nearest even, NaN stays NaN
    return __builtin_bit_cast(uint16_t, __bf16(v));
  }
};

// Eight consecutive elements widened to fp32: one or two 16-byte loads where the
// caller knows the address to be 16-byte aligned, else eight loads.
template <class T, bool ALIGNED>
__device__ __forceinline__ void load8(const typename T::raw* p, float (&f)[8]) {
  if constexpr (!ALIGNED) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = T::widen(p[i]);
  } else if constexpr (sizeof(typename T::raw) == 4) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w;
    f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
  } else {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = T::widen(uint16_t(w[i] & 0xFFFFu));
      f[2 * i + 1] = T::widen(uint16_t(w[i] >> 16));
    }
  }
}

template <class T, bool ALIGNED>
__device__ __forceinline__ void store8(typename T::raw* p, const float (&f)[8]) {
  if constexpr (!ALIGNED) {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = T::narrow(f[i]);
  } else if constexpr (sizeof(typename T::raw) == 4) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = uint32_t(T::narrow(f[2 * i])) | uint32_t(T::narrow(f[2 * i + 1])) << 16;
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// Calls f with the element type of a SEEDQ_* type code (checked by the caller).
template <class F>
inline hipError_t with_type(int type, F f) {
  switch (type) {
    case SEEDQ_F32: return f(F32{});
    case SEEDQ_F16: return f(F16{});
    case SEEDQ_BF16: return f(BF16{});
    default: return hipErrorInvalidValue;
  }
}

// 16-byte aligned rows of elements of `size` bytes.
inline bool rows_aligned(const void* p, int64_t ld, size_t size) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (uint64_t(ld) * size) % 16 == 0;
}

}  // namespace seedq
