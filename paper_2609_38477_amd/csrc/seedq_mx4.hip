// Microscaled 4-bit floats: the quantiser and the decoder.
//
// Both are one pass over the weights, bound by memory. A lane holds eight consecutive
// columns, which are one word of codes, and a block lies in four neighbouring lanes, so its
// largest weight is found without LDS. The block's exponent is that weight's exponent
// field less 2, as a number of its own and as the scale of the conversions both ways: the
// conversion instructions take a power of two by its exponent field alone, 0 standing for
// 2^-127, round to nearest even and saturate, which is the definition's rounding. 4096 x
// 14336 bf16 is coded in 25 to 28 us and decoded in 23 (5.3 to 6.4 TB/s of weights and codes,
// some of them from the last-level cache), 1024 x 4096 fp32 in 4.9 and 6.6.
#include "seedq_mx4_internal.h"
#include "seedq_mx4_device.h"

namespace seedq {
namespace {

typedef float floatx2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// A wave: 64 words of one row.
template <class T>
__global__ void __launch_bounds__(kThreads)
quantize_kernel(const typename T::raw* __restrict__ W, int64_t ldw, Mx4 q, uint32_t per_row,
                int64_t total) {
  uint32_t* __restrict__ codes = const_cast<uint32_t*>(q.codes);
  uint8_t* __restrict__ scale = const_cast<uint8_t*>(q.scale);
  const int lane = int(threadIdx.x & 63);
  const int64_t job = int64_t(blockIdx.x) * kWaves + (threadIdx.x >> 6);
  if (job >= total) return;
  const int64_t r = int64_t(uint32_t(job) / per_row);
  const int64_t word = int64_t(uint32_t(job) % per_row) * 64 + lane, c = word * 8;
  float w[8] = {};
  if (c < q.ncols) load8<T>(W + r * ldw + c, w);
  uint32_t big = 0;   // the largest pattern without sign
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __builtin_bit_cast(uint32_t, w[i]) & 0x7FFFFFFFu;
    big = b > big ? b : big;
  }
  big = lanes_reduce<4>(big, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
  const bool finite = big < 0x7F800000u;
  const uint32_t field = big >> 23, e = field > 2 ? field - 2 : 0;
  const float s = mx_scale(e);
  uint32_t code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, w[0], w[1], s, 0);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, w[2], w[3], s, 1);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, w[4], w[5], s, 2);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, w[6], w[7], s, 3);
  if (word < q.row_words) codes[r * q.row_words + word] = finite ? code : 0u;   // 0 after the last column
  if (c < q.ncols && (lane & 3) == 0) scale[r * q.nblocks + (word >> 2)] = finite ? uint8_t(e) : uint8_t(255);
}

template <class T>
__global__ void __launch_bounds__(kThreads)
dequantize_kernel(Mx4 q, uint32_t per_row, int64_t total, typename T::raw* __restrict__ W, int64_t ldw) {
  const int lane = int(threadIdx.x & 63);
  const int64_t job = int64_t(blockIdx.x) * kWaves + (threadIdx.x >> 6);
  if (job >= total) return;
  const int64_t r = int64_t(uint32_t(job) / per_row);
  const int64_t word = int64_t(uint32_t(job) % per_row) * 64 + lane, c = word * 8;
  if (c >= q.ncols) return;
  const uint32_t code = q.codes[r * q.row_words + word];
  const float s = mx_scale(q.scale[r * q.nblocks + (word >> 2)]);
  const floatx2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 0);
  const floatx2 p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 1);
  const floatx2 p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 2);
  const floatx2 p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 3);
  const float f[8] = {p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
  store8<T>(W + r * ldw + c, f);
}

// A wave for every 64 words.
struct Jobs {
  uint32_t per_row;
  int64_t total;
  unsigned grid;
};
Jobs jobs(int64_t nrows, int64_t words) {
  Jobs j;
  j.per_row = uint32_t((words + 63) / 64);
  j.total = nrows * int64_t(j.per_row);   // at most one for each block of 8: below 2^31
  j.grid = unsigned((j.total + kWaves - 1) / kWaves);
  return j;
}

}  // namespace

hipError_t launch_mx4_quantize(const void* d_W, int type, int64_t ldw, const Mx4& q,
                               hipStream_t stream) {
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    using raw = typename T::raw;
    for (int64_t r = 0; r < q.nrows; r += kMaxRows) {
      const Mx4 part = q.rows(r);
      const Jobs j = jobs(part.nrows, q.row_words);
      hipLaunchKernelGGL(quantize_kernel<T>, dim3(j.grid), dim3(kThreads), 0, stream,
                         static_cast<const raw*>(d_W) + r * ldw, ldw, part, j.per_row, j.total);
    }
    return hipGetLastError();
  });
}

hipError_t launch_mx4_dequantize(const Mx4& q, void* d_W_hat, int type, int64_t ldw,
                                 hipStream_t stream) {
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    using raw = typename T::raw;
    for (int64_t r = 0; r < q.nrows; r += kMaxRows) {
      const Mx4 part = q.rows(r);
      const Jobs j = jobs(part.nrows, q.ncols / kC);
      hipLaunchKernelGGL(dequantize_kernel<T>, dim3(j.grid), dim3(kThreads), 0, stream, part,
                         j.per_row, j.total, static_cast<raw*>(d_W_hat) + r * ldw, ldw);
    }
    return hipGetLastError();
  });
}

}  // namespace seedq
