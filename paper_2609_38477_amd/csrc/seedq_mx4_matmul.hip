// Products of two matrices of microscaled 4-bit floats on the matrix core, which takes the
// codes and the blocks' exponents as they lie in memory: lane l of a 32x32x64 product holds
// the 16 bytes of block l / 32 of row l % 32 and that block's exponent.
#include <algorithm>

#include "seedq_mx4_internal.h"
#include "seedq_ops_device.h"

namespace seedq {
namespace {

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ void store_y(void* y, int ytype, int64_t at, float v) {
  if (ytype == SEEDQ_F32) static_cast<float*>(y)[at] = v;
  else static_cast<uint16_t*>(y)[at] = ytype == SEEDQ_F16 ? F16::narrow(v) : BF16::narrow(v);
}

__device__ __forceinline__ intx8 fp4_operand(uint32x4 c) {
  return intx8{int(c[0]), int(c[1]), int(c[2]), int(c[3]), 0, 0, 0, 0};
}

// A wave makes 32 x 32 of Y.
__global__ void __launch_bounds__(256)
matmul_kernel(Mx4 a, Mx4 b, void* __restrict__ y, int ytype, int64_t ldy) {
  const int lane = int(threadIdx.x & 63), n = lane & 31, kg = lane >> 5;
  const int64_t j0 = (int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6)) * 32, j = std::min(j0 + n, b.nrows - 1);
  if (j0 >= b.nrows) return;
  for (int64_t i0 = int64_t(blockIdx.y) * 32; i0 < a.nrows; i0 += int64_t(gridDim.y) * 32) {
    const int64_t i = std::min(i0 + n, a.nrows - 1);
    floatx16 acc = {};
    for (int64_t k = kg; k < b.nblocks + kg; k += 2) {
      uint32x4 ca = {0u, 0u, 0u, 0u}, cb = {0u, 0u, 0u, 0u};
      int sa = 0, sb = 0;
      if (k < b.nblocks) {
        ca = *reinterpret_cast<const uint32x4*>(a.codes + i * a.row_words + k * 4);
        cb = *reinterpret_cast<const uint32x4*>(b.codes + j * b.row_words + k * 4);
        sa = a.scale[i * a.nblocks + k];
        sb = b.scale[j * b.nblocks + k];
      }
      acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fp4_operand(ca), fp4_operand(cb), acc, 4, 4, 0,
                                                            sa, 0, sb);
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int64_t row = i0 + 8 * (e >> 2) + 4 * kg + (e & 3);
      if (row < a.nrows && j0 + n < b.nrows) store_y(y, ytype, row * ldy + j0 + n, acc[e]);
    }
  }
}

}  // namespace

size_t mx4_matmul_workspace_bytes(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_mx4_matmul(const Mx4& a, const Mx4& all, void* d_y, int ytype, int64_t ldy, void*,
                             hipStream_t stream) {
  for (int64_t r = 0; r < all.nrows; r += kMaxRows) {
    const Mx4 b = all.rows(r);
    hipLaunchKernelGGL(matmul_kernel,
                       dim3(unsigned((b.nrows + 127) / 128), unsigned(std::min<int64_t>((a.nrows + 31) / 32, 4096))),
                       dim3(256), 0, stream, a, b, static_cast<char*>(d_y) + r * (ytype == SEEDQ_F32 ? 4 : 2),
                       ytype, ldy);
  }
  return hipGetLastError();
}

}  // namespace seedq
