// Weights in 4 bits with group scales: the quantiser and the decoder.
//
// Both are one pass over the weights, bound by memory. A lane holds eight
// consecutive columns, which are one word of codes: a wave covers 512 columns of a
// row, so every group (32 to 512 columns) lies in 4 to 64 neighbouring lanes of
// one wave and its extremes are found with shuffles.
#include "seedq_ops_device.h"

namespace seedq {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr float kMaxHalf = 65504.0f;

// rne(fl32(w / s)). The product with the reciprocal is within 2e-6 of the quotient
// (at most 16 where it is not clamped), so the division is only taken near a tie.
__device__ __forceinline__ float rounded_quotient(float w, float s, float inv) {
  const float t = w * inv;
  float q = rintf(t);
  if (__builtin_expect(fabsf(t - q) > 0.49999f, 0)) q = rintf(w / s);
  return q;
}

template <class T, bool ZEROS>
__global__ void __launch_bounds__(kThreads)
quantize_kernel(const typename T::raw* __restrict__ W, int64_t ldw, Q4 q, uint32_t tiles,
                int64_t total) {
  uint32_t* __restrict__ codes = const_cast<uint32_t*>(q.codes);
  uint16_t* __restrict__ scale = const_cast<uint16_t*>(q.scale);
  uint8_t* __restrict__ zero = const_cast<uint8_t*>(q.zero);
  const int64_t ncols = q.ncols;
  const int gshift = q.gshift;
  const int lane = int(threadIdx.x & 63);
  const int64_t job = int64_t(blockIdx.x) * kWaves + (threadIdx.x >> 6);
  if (job >= total) return;
  const int64_t r = int64_t(uint32_t(job) / tiles);
  const int64_t word = int64_t(uint32_t(job) % tiles) * 64 + lane, c = word * 8;
  float w[8] = {};
  if (c < ncols) load8<T>(W + r * ldw + c, w);
  float lo = 0.f, hi = 0.f;
  uint32_t big = 0;   // the largest pattern without sign: above 0x7F7FFFFF it is not finite
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo = fminf(lo, w[i]);
    hi = fmaxf(hi, w[i]);
    const uint32_t b = __builtin_bit_cast(uint32_t, w[i]) & 0x7FFFFFFFu;
    big = b > big ? b : big;
  }
  const int lanes = 1 << (gshift - 3);
  for (int d = 1; d < lanes; d <<= 1) {
    if (ZEROS) {
      lo = fminf(lo, __shfl_xor(lo, d, 64));
      hi = fmaxf(hi, __shfl_xor(hi, d, 64));
    }
    const uint32_t b = __shfl_xor(big, d, 64);
    big = b > big ? b : big;
  }
  const bool finite = big < 0x7F800000u;
  const float span = ZEROS ? hi - lo : __builtin_bit_cast(float, big);
  const _Float16 sh = _Float16(fminf(span / (ZEROS ? 15.0f : 7.0f), kMaxHalf));
  const float s = float(sh);
  const float inv = s > 0.f ? 1.0f / s : 0.f;
  float z = 8.f;
  if (ZEROS) z = s > 0.f ? fminf(fmaxf(rintf(-lo / s), 0.f), 15.f) : 0.f;
  uint32_t code = 0;
  if (finite && c < ncols) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = s > 0.f ? rounded_quotient(w[i], s, inv) : 0.f;
      code |= uint32_t(fminf(fmaxf(t + z, 0.f), 15.f)) << (4 * i);
    }
  }
  if (word < q.row_words) codes[r * q.row_words + word] = code;   // zero after the last column
  if (c < ncols && (lane & (lanes - 1)) == 0) {
    const int64_t g = r * q.ngroups + (c >> gshift);
    scale[g] = finite ? __builtin_bit_cast(uint16_t, sh) : uint16_t(0x7E00);
    if (ZEROS) zero[g] = finite ? uint8_t(z) : uint8_t(0);
  }
}

template <class T>
__global__ void __launch_bounds__(kThreads)
dequantize_kernel(Q4 q, uint32_t tiles, int64_t total, typename T::raw* __restrict__ W,
                  int64_t ldw) {
  const int lane = int(threadIdx.x & 63);
  const int64_t job = int64_t(blockIdx.x) * kWaves + (threadIdx.x >> 6);
  if (job >= total) return;
  const int64_t r = int64_t(uint32_t(job) / tiles);
  const int64_t word = int64_t(uint32_t(job) % tiles) * 64 + lane, c = word * 8;
  if (c >= q.ncols) return;
  const uint32_t code = q.codes[r * q.row_words + word];
  const int64_t g = r * q.ngroups + (c >> q.gshift);
  const float s = F16::widen(q.scale[g]);
  const float z = q.zero ? float(q.zero[g] & 15) : 8.f;
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = (float((code >> (4 * i)) & 15u) - z) * s;
  store8<T>(W + r * ldw + c, f);
}

// Jobs of one wave: 64 words of one row.
struct Jobs {
  uint32_t tiles;
  int64_t total;
  unsigned grid;
};
Jobs jobs(int64_t nrows, int64_t words) {
  Jobs j;
  j.tiles = uint32_t((words + 63) / 64);
  j.total = nrows * int64_t(j.tiles);   // at most one for each block of 8: below 2^31
  j.grid = unsigned((j.total + kWaves - 1) / kWaves);
  return j;
}

}  // namespace

hipError_t launch_q4_quantize(const void* d_W, int type, int64_t ldw, const Q4& q,
                              hipStream_t stream) {
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    using raw = typename T::raw;
    for (int64_t r = 0; r < q.nrows; r += kMaxRows) {
      const Q4 part = q.rows(r);
      const Jobs j = jobs(part.nrows, q.row_words);
      auto launch = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(j.grid), dim3(kThreads), 0, stream,
                           static_cast<const raw*>(d_W) + r * ldw, ldw, part, j.tiles, j.total);
      };
      q.zero ? launch(quantize_kernel<T, true>) : launch(quantize_kernel<T, false>);
    }
    return hipGetLastError();
  });
}

hipError_t launch_q4_dequantize(const Q4& q, void* d_W_hat, int type, int64_t ldw,
                                hipStream_t stream) {
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    using raw = typename T::raw;
    for (int64_t r = 0; r < q.nrows; r += kMaxRows) {
      const Q4 part = q.rows(r);
      const Jobs j = jobs(part.nrows, q.ncols / kC);
      hipLaunchKernelGGL(dequantize_kernel<T>, dim3(j.grid), dim3(kThreads), 0, stream, part, j.tiles,
                         j.total, static_cast<raw*>(d_W_hat) + r * ldw, ldw);
    }
    return hipGetLastError();
  });
}

}  // namespace seedq
