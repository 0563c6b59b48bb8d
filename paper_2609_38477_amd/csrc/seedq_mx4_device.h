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

// Partial sums [splits][n][m], those of one place added in order, to rows of y. A thread takes
// four neighbours. What bounds it is the way to the loads and, of many sums, their memory: a
// product of 512 x 4096 places whose two or three sums it adds takes 21.4 us with it and 24.5
// with a thread a place; of 8 x 8192 places and eight sums as long as that.
template <int NT>
static __global__ void __launch_bounds__(NT)
join_kernel(const float* __restrict__ partial, int splits, int64_t n, int64_t m, void* __restrict__ y,
            int ytype, int64_t ldy) {
  typedef float floatx4_at4 __attribute__((ext_vector_type(4), aligned(4)));
  typedef uint32_t uint32x2_at2 __attribute__((ext_vector_type(2), aligned(2)));
  const int64_t i = blockIdx.y, j = (int64_t(blockIdx.x) * NT + threadIdx.x) * 4;
  if (j >= m) return;
  const float* p = partial + i * m + j;
  const int64_t at = i * ldy + j;
  if (j + 4 <= m) {
    floatx4_at4 sum = {};
#pragma unroll 4
    for (int s = 0; s < splits; ++s) sum += *reinterpret_cast<const floatx4_at4*>(p + s * n * m);
    if (ytype == SEEDQ_F32) {
      *reinterpret_cast<floatx4_at4*>(static_cast<float*>(y) + at) = sum;
    } else {
      uint32_t v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = ytype == SEEDQ_F16 ? F16::narrow(sum[k]) : BF16::narrow(sum[k]);
      *reinterpret_cast<uint32x2_at2*>(static_cast<uint16_t*>(y) + at) =
          uint32x2_at2{v[0] | v[1] << 16, v[2] | v[3] << 16};
    }
    return;
  }
  for (int64_t k = 0; k < m - j; ++k) {
    float sum = 0.f;
    for (int s = 0; s < splits; ++s) sum += p[s * n * m + k];
    store_y(y, ytype, at + k, sum);
  }
}

// Small workgroups where there are few sums, so that more CUs have some.
inline void launch_join(const float* partial, int splits, int64_t n, int64_t m, void* y, int ytype, int64_t ldy,
                        hipStream_t stream) {
  const auto go = [&](auto kern, int threads) {
    hipLaunchKernelGGL(kern, dim3(unsigned((m + 4 * threads - 1) / (4 * threads)), unsigned(n)), dim3(threads), 0,
                       stream, partial, splits, n, m, y, ytype, ldy);
  };
  if ((m + 1023) / 1024 * n < 512) go(join_kernel<64>, 64);
  else go(join_kernel<256>, 256);
}

}  // namespace seedq
