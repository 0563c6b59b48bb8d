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

typedef uint32_t uint32x4 __attribute__((ext_vector_type(4)));
// 16 bytes at any element: global loads and stores of vectors need no alignment here.
typedef uint32x4 uint32x4_any __attribute__((aligned(2)));

__device__ __forceinline__ uint32x4 load16(const void* p) {
  return *static_cast<const uint32x4_any*>(p);
}
__device__ __forceinline__ void store16(void* p, uint32x4 v) { *static_cast<uint32x4_any*>(p) = v; }

// The elements of a vector in fp32, and back.
template <class T>
constexpr int kPerVector = 16 / sizeof(typename T::raw);

template <class T>
__device__ __forceinline__ void widen(uint32x4 v, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = v[i];
    if constexpr (kPerVector<T> == 4) {
      f[i] = __builtin_bit_cast(float, w);
    } else {
      f[2 * i] = T::widen(uint16_t(w & 0xFFFFu));
      f[2 * i + 1] = T::widen(uint16_t(w >> 16));
    }
  }
}
template <class T>
__device__ __forceinline__ uint32x4 narrow(const float* f) {
  uint32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (kPerVector<T> == 4) v[i] = __builtin_bit_cast(uint32_t, f[i]);
    else v[i] = uint32_t(T::narrow(f[2 * i])) | uint32_t(T::narrow(f[2 * i + 1])) << 16;
  }
  return v;
}

// Eight consecutive elements.
template <class T>
__device__ __forceinline__ void load8(const typename T::raw* p, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i += kPerVector<T>) widen<T>(load16(p + i), f + i);
}
template <class T>
__device__ __forceinline__ void store8(typename T::raw* p, const float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i += kPerVector<T>) store16(p + i, narrow<T>(f + i));
}

// f over `LANES` neighbouring lanes (a power of two), the result in all of them; f
// commutes, so it is the same in all. Steps within 16 lanes are data-parallel moves (the
// mirrored ones meet a half whose lanes all hold the same), those across exchange rows.
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
  return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), CTRL, 0xF, 0xF, true));
}
template <class V, class F>
__device__ __forceinline__ V apart(V v, F f) {   // f on the 32-bit words of v
  static_assert(sizeof(V) == 4 || sizeof(V) == 8, "one or two words");
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(V, f(__builtin_bit_cast(uint32_t, v)));
  } else {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(V, uint64_t(f(uint32_t(u))) | uint64_t(f(uint32_t(u >> 32))) << 32);
  }
}
// One step: from groups of LANES / 2 lanes to groups of LANES.
template <int LANES, class V, class F>
__device__ __forceinline__ V lanes_step(V v, F f) {
  if constexpr (LANES == 2) return f(v, apart(v, [](uint32_t w) { return moved<0xB1>(w); }));
  if constexpr (LANES == 4) return f(v, apart(v, [](uint32_t w) { return moved<0x4E>(w); }));
  if constexpr (LANES == 8) return f(v, apart(v, [](uint32_t w) { return moved<0x141>(w); }));
  if constexpr (LANES == 16) return f(v, apart(v, [](uint32_t w) { return moved<0x140>(w); }));
  if constexpr (LANES == 32)
    return f(apart(v, [](uint32_t w) { return __builtin_amdgcn_permlane16_swap(w, w, false, false)[0]; }),
             apart(v, [](uint32_t w) { return __builtin_amdgcn_permlane16_swap(w, w, false, false)[1]; }));
  if constexpr (LANES == 64)
    return f(apart(v, [](uint32_t w) { return __builtin_amdgcn_permlane32_swap(w, w, false, false)[0]; }),
             apart(v, [](uint32_t w) { return __builtin_amdgcn_permlane32_swap(w, w, false, false)[1]; }));
}
template <int LANES = 64, class V, class F>
__device__ __forceinline__ V lanes_reduce(V v, F f) {
  if constexpr (LANES >= 2) v = lanes_step<2>(v, f);
  if constexpr (LANES >= 4) v = lanes_step<4>(v, f);
  if constexpr (LANES >= 8) v = lanes_step<8>(v, f);
  if constexpr (LANES >= 16) v = lanes_step<16>(v, f);
  if constexpr (LANES >= 32) v = lanes_step<32>(v, f);
  if constexpr (LANES >= 64) v = lanes_step<64>(v, f);
  return v;
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

}  // namespace seedq
