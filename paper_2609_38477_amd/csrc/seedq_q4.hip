// Weights in 4 bits with group scales: the quantiser and the decoder.
//
// Both are one pass over the weights, bound by memory. A lane holds eight
// consecutive columns, which are one word of codes: a wave covers 512 columns of a
// row, so every group (32 to 512 columns) lies in 4 to 64 neighbouring lanes of
// one wave and its extremes are found without LDS. At 8192 x 28672 bf16 in groups of 128 the
// quantiser takes 129 us (4.6 TB/s) and the decoder 109 us (5.4 TB/s, the rate of a large
// copy); at 4096 x 14336 fp32 47 us (5.7 TB/s, from the last-level cache in part) and 55 us.
// What is left over the copy's rate in 16 bits is the arithmetic, some 12 operations a
// weight, more with zero points: 4096 x 14336 bf16 in groups of 64 takes 41 us with them.
#include "seedq_ops_device.h"

namespace seedq {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr float kMaxHalf = 65504.0f;

// f over the `lanes` (4 to 64) neighbouring lanes of a group, the result in all of them.
template <class V, class F>
__device__ __forceinline__ V group_reduce(V v, int lanes, F f) {
  v = lanes_reduce<4>(v, f);
  if (lanes > 4) v = lanes_step<8>(v, f);
  if (lanes > 8) v = lanes_step<16>(v, f);
  if (lanes > 16) v = lanes_step<32>(v, f);
  if (lanes > 32) v = lanes_step<64>(v, f);
  return v;
}

// rne(fl32(w / s)) for eight weights. The product with the reciprocal is within 2e-6 of the
// quotient (at most 16 where it is not clamped), so the divisions are only taken where
// one lies next to a tie.
__device__ __forceinline__ void rounded_quotients(const float (&w)[8], float s, float inv, float (&q)[8]) {
  float off = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float t = w[i] * inv;
    q[i] = rintf(t);
    off = fmaxf(off, fabsf(t - q[i]));
  }
  if (__builtin_expect(off > 0.49999f, 0))
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = rintf(w[i] / s);
}

// The columns of a wave: TILES pieces of 64 words of one row, read before the first is
// worked on.
template <class T, bool ZEROS, int TILES>
__global__ void __launch_bounds__(kThreads)
quantize_kernel(const typename T::raw* __restrict__ W, int64_t ldw, Q4 q, uint32_t per_row,
                int64_t total) {
  uint32_t* __restrict__ codes = const_cast<uint32_t*>(q.codes);
  uint16_t* __restrict__ scale = const_cast<uint16_t*>(q.scale);
  uint8_t* __restrict__ zero = const_cast<uint8_t*>(q.zero);
  const int lane = int(threadIdx.x & 63);
  const int64_t job = int64_t(blockIdx.x) * kWaves + (threadIdx.x >> 6);
  if (job >= total) return;
  const int64_t r = int64_t(uint32_t(job) / per_row);
  const int64_t word0 = int64_t(uint32_t(job) % per_row) * (64 * TILES) + lane;
  float all[TILES][8];
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    const int64_t c = (word0 + 64 * t) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) all[t][i] = 0.f;
    if (c < q.ncols) load8<T>(W + r * ldw + c, all[t]);
  }
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    const int64_t word = word0 + 64 * t, c = word * 8;
    const float(&w)[8] = all[t];
    float lo = 0.f, hi = 0.f;
    uint32_t big = 0;   // the largest pattern without sign: above 0x7F7FFFFF it is not finite
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo = fminf(lo, w[i]);
      hi = fmaxf(hi, w[i]);
      const uint32_t b = __builtin_bit_cast(uint32_t, w[i]) & 0x7FFFFFFFu;
      big = b > big ? b : big;
    }
    const int lanes = 1 << (q.gshift - 3);
    if (ZEROS) {
      lo = group_reduce(lo, lanes, [](float x, float y) { return fminf(x, y); });
      hi = group_reduce(hi, lanes, [](float x, float y) { return fmaxf(x, y); });
    }
    big = group_reduce(big, lanes, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
    const bool finite = big < 0x7F800000u;
    const float span = ZEROS ? hi - lo : __builtin_bit_cast(float, big);
    const _Float16 sh = _Float16(fminf(span / (ZEROS ? 15.0f : 7.0f), kMaxHalf));
    const float s = float(sh);
    const float inv = s > 0.f ? 1.0f / s : 0.f;
    float z = 8.f;
    if (ZEROS) z = s > 0.f ? fminf(fmaxf(rintf(-lo / s), 0.f), 15.f) : 0.f;
    uint32_t code = 0;
    if (finite && c < q.ncols) {
      float v[8];
      rounded_quotients(w, s, inv, v);   // all 0 where s is
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __builtin_amdgcn_fmed3f(v[i], -z, 15.f - z);
      // half a word is a whole number below 2^16 in fp32; the zero points join at the end
      const float low = fmaf(fmaf(fmaf(v[3], 16.f, v[2]), 16.f, v[1]), 16.f, v[0]);
      const float high = fmaf(fmaf(fmaf(v[7], 16.f, v[6]), 16.f, v[5]), 16.f, v[4]);
      code = uint32_t(int(low)) + (uint32_t(int(high)) << 16) + uint32_t(z) * 0x11111111u;
    }
    if (word < q.row_words) codes[r * q.row_words + word] = code;   // zero after the last column
    if (c < q.ncols && (lane & (lanes - 1)) == 0) {
      const int64_t g = r * q.ngroups + (c >> q.gshift);
      scale[g] = finite ? __builtin_bit_cast(uint16_t, sh) : uint16_t(0x7E00);
      if (ZEROS) zero[g] = finite ? uint8_t(z) : uint8_t(0);
    }
  }
}

template <class T, int TILES>
__global__ void __launch_bounds__(kThreads)
dequantize_kernel(Q4 q, uint32_t per_row, int64_t total, typename T::raw* __restrict__ W,
                  int64_t ldw) {
  const int lane = int(threadIdx.x & 63);
  const int64_t job = int64_t(blockIdx.x) * kWaves + (threadIdx.x >> 6);
  if (job >= total) return;
  const int64_t r = int64_t(uint32_t(job) / per_row);
  const int64_t word0 = int64_t(uint32_t(job) % per_row) * (64 * TILES) + lane;
  uint32_t code[TILES];
  uint16_t scale[TILES];
  uint8_t zero[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    const int64_t word = word0 + 64 * t;
    if (word * 8 >= q.ncols) break;
    code[t] = q.codes[r * q.row_words + word];
    const int64_t g = r * q.ngroups + (word * 8 >> q.gshift);
    scale[t] = q.scale[g];
    zero[t] = q.zero ? q.zero[g] : uint8_t(8);
  }
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    const int64_t c = (word0 + 64 * t) * 8;
    if (c >= q.ncols) break;
    const float s = F16::widen(scale[t]), z = float(zero[t] & 15);
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float((code[t] >> (4 * i)) & 15u) - z) * s;
    store8<T>(W + r * ldw + c, f);
  }
}

// A wave for every `tiles` pieces of 64 words.
struct Jobs {
  uint32_t per_row;
  int64_t total;
  unsigned grid;
};
Jobs jobs(int64_t nrows, int64_t words, int tiles) {
  Jobs j;
  j.per_row = uint32_t((words + 64 * tiles - 1) / (64 * tiles));
  j.total = nrows * int64_t(j.per_row);   // at most one for each block of 8: below 2^31
  j.grid = unsigned((j.total + kWaves - 1) / kWaves);
  return j;
}

// Two pieces a wave for many weights of 16 bits (8192 x 28672 bf16 decoded in 109 us, one
// piece 114, four 109), one for few and in fp32 (4096 x 14336 decoded in 55 us, two 64;
// 1024 x 4096 coded in 6.3, two 7.2).
int tiles_of(int64_t nrows, int64_t words, size_t size) {
  return size == 2 && nrows * words >= int64_t(1) << 21 ? 2 : 1;
}

}  // namespace

hipError_t launch_q4_quantize(const void* d_W, int type, int64_t ldw, const Q4& q,
                              hipStream_t stream) {
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    using raw = typename T::raw;
    for (int64_t r = 0; r < q.nrows; r += kMaxRows) {
      const Q4 part = q.rows(r);
      const int tiles = tiles_of(part.nrows, q.row_words, sizeof(raw));
      const Jobs j = jobs(part.nrows, q.row_words, tiles);
      auto launch = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(j.grid), dim3(kThreads), 0, stream,
                           static_cast<const raw*>(d_W) + r * ldw, ldw, part, j.per_row, j.total);
      };
      if (tiles == 1) q.zero ? launch(quantize_kernel<T, true, 1>) : launch(quantize_kernel<T, false, 1>);
      else q.zero ? launch(quantize_kernel<T, true, 2>) : launch(quantize_kernel<T, false, 2>);
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
      const int tiles = tiles_of(part.nrows, q.ncols / kC, sizeof(raw));
      const Jobs j = jobs(part.nrows, q.ncols / kC, tiles);
      auto launch = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(j.grid), dim3(kThreads), 0, stream, part, j.per_row, j.total,
                           static_cast<raw*>(d_W_hat) + r * ldw, ldw);
      };
      tiles == 1 ? launch(dequantize_kernel<T, 1>) : launch(dequantize_kernel<T, 2>);
    }
    return hipGetLastError();
  });
}

}  // namespace seedq
