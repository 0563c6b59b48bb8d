// Products of a matrix of microscaled 4-bit floats with vectors of 16 or 32 bits, straight
// from the codes.
#include <algorithm>

#include "seedq_mx4_internal.h"
#include "seedq_ops_device.h"

namespace seedq {
namespace {

typedef float floatx2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void store_y(void* y, int ytype, int64_t at, float v) {
  if (ytype == SEEDQ_F32) static_cast<float*>(y)[at] = v;
  else static_cast<uint16_t*>(y)[at] = ytype == SEEDQ_F16 ? F16::narrow(v) : BF16::narrow(v);
}

// A wave a row and four vectors at a time: lane l takes the row's words l, l + 64, ...
template <class X>
__global__ void __launch_bounds__(256)
gemv_kernel(Mx4 q, int64_t nvec, const typename X::raw* __restrict__ x, int64_t ldx,
            void* __restrict__ y, int ytype, int64_t ldy) {
  const int lane = int(threadIdx.x & 63);
  const int64_t r = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (r >= q.nrows) return;
  const int64_t words = q.ncols / kC;
  for (int64_t v0 = int64_t(blockIdx.y) * 4; v0 < nvec; v0 += int64_t(gridDim.y) * 4) {
    float acc[4] = {};
    for (int64_t w = lane; w < words; w += 64) {
      const uint32_t code = q.codes[r * q.row_words + w];
      const float s = __builtin_bit_cast(float, uint32_t(q.scale[r * q.nblocks + (w >> 2)]) << 23);
      const floatx2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 0),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 1),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 2),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 3)};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float f[8];
        load8<X>(x + std::min(v0 + i, nvec - 1) * ldx + w * kC, f);
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[i] = fmaf(p[k / 2][k % 2], f[k], acc[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float total = lanes_reduce(acc[i], [](float a, float b) { return a + b; });
      if (lane == 0 && v0 + i < nvec) store_y(y, ytype, (v0 + i) * ldy + r, total);
    }
  }
}

}  // namespace

size_t mx4_gemv_workspace_bytes(int64_t, int64_t, int64_t, int) { return 0; }

hipError_t launch_mx4_gemv(const Mx4& all, int64_t nvec, const void* d_x, int xtype, int64_t ldx,
                           void* d_y, int ytype, int64_t ldy, void*, hipStream_t stream) {
  return with_type(xtype, [&](auto t) {
    using X = decltype(t);
    for (int64_t r = 0; r < all.nrows; r += kMaxRows) {
      const Mx4 q = all.rows(r);
      hipLaunchKernelGGL(gemv_kernel<X>,
                         dim3(unsigned((q.nrows + 3) / 4), unsigned(std::min<int64_t>((nvec + 3) / 4, 4096))),
                         dim3(256), 0, stream, q, nvec, static_cast<const typename X::raw*>(d_x), ldx,
                         static_cast<char*>(d_y) + r * (ytype == SEEDQ_F32 ? 4 : 2), ytype, ldy);
    }
    return hipGetLastError();
  });
}

}  // namespace seedq
