// Products of a 4-bit matrix with vectors, straight from the codes.
#include <algorithm>

#include "seedq_ops_device.h"

namespace seedq {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// One wave a row, NV vectors at a time: lanes over the row's words, the eight
// products of a word summed before the scale enters, then a tree over the lanes.
template <class X, class Y, bool ALIGNED, int NV>
__global__ void __launch_bounds__(kThreads)
gemv_kernel(Q4 q, int64_t nvec, const typename X::raw* __restrict__ x, int64_t ldx,
            typename Y::raw* __restrict__ y, int64_t ldy) {
  const int lane = int(threadIdx.x & 63);
  const int64_t r = int64_t(blockIdx.x) * kWaves + (threadIdx.x >> 6);
  if (r >= q.nrows) return;
  const uint32_t* codes = q.codes + r * q.row_words;
  const int64_t words = q.ncols / kC;
  for (int64_t v0 = int64_t(blockIdx.y) * NV; v0 < nvec; v0 += int64_t(gridDim.y) * NV) {
    float sum[NV] = {};
    for (int64_t w = lane; w < words; w += 64) {
      const uint32_t code = codes[w];
      const int64_t g = r * q.ngroups + ((w * 8) >> q.gshift);
      const float s = F16::widen(q.scale[g]);
      const float z = q.zero ? float(q.zero[g] & 15) : 8.f;
      float u[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = float((code >> (4 * i)) & 15u) - z;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float f[8];
        const int64_t vv = std::min(v0 + v, nvec - 1);
        load8<X, ALIGNED>(x + vv * ldx + w * 8, f);
        float t = u[0] * f[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) t = fmaf(u[i], f[i], t);
        sum[v] = fmaf(s, t, sum[v]);
      }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) sum[v] += __shfl_xor(sum[v], d, 64);
      if (lane == 0 && v0 + v < nvec) y[(v0 + v) * ldy + r] = Y::narrow(sum[v]);
    }
  }
}

}  // namespace

size_t q4_gemv_workspace_bytes(int64_t, int64_t, int64_t, int) { return 0; }

hipError_t launch_q4_gemv(const Q4& q, int64_t nvec, const void* d_x, int xtype, int64_t ldx,
                          void* d_y, int ytype, int64_t ldy, void*, hipStream_t stream) {
  return with_type(xtype, [&](auto tx) {
    using X = decltype(tx);
    auto launch = [&](auto ty) {
      using Y = decltype(ty);
      const dim3 grid(unsigned((q.nrows + kWaves - 1) / kWaves),
                      unsigned(std::min<int64_t>((nvec + 3) / 4, 65535)));
      auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, grid, dim3(kThreads), 0, stream, q, nvec,
                           static_cast<const typename X::raw*>(d_x), ldx,
                           static_cast<typename Y::raw*>(d_y), ldy);
      };
      rows_aligned(d_x, ldx, sizeof(typename X::raw)) ? go(gemv_kernel<X, Y, true, 4>)
                                                      : go(gemv_kernel<X, Y, false, 4>);
      return hipGetLastError();
    };
    return ytype == SEEDQ_F32 ? launch(F32{}) : launch(tx);
  });
}

}  // namespace seedq
