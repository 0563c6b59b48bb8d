// Log probabilities of given tokens with entropy and top alternatives, and their
// gradient at the logits.
#include <algorithm>

#include "seedq_ops_device.h"

namespace seedq {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr float kInf = __builtin_inff();

template <class V, class F>
__device__ V block_reduce(V v, V* shared, F f) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v = f(v, __shfl_xor(v, d, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
  __syncthreads();
  v = shared[0];
  for (int w = 1; w < int(blockDim.x >> 6); ++w) v = f(v, shared[w]);
  return v;
}

// Order of alternatives in one number: the value's pattern made monotonic (-0 is
// 0), then the lower token first. 0 stands for none.
__device__ __forceinline__ unsigned long long order_key(float x, uint32_t v) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
  const uint32_t k = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (static_cast<unsigned long long>(k) << 32) | (0xFFFFFFFFu - v);
}
__device__ __forceinline__ float key_value(unsigned long long key) {
  const uint32_t k = uint32_t(key >> 32);
  return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ uint32_t key_token(unsigned long long key) {
  return 0xFFFFFFFFu - uint32_t(key);
}

// One workgroup a row: the maximum, the sums, then one pass for each alternative.
template <class T>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(LogprobArgs a) {
  __shared__ double sd[kWaves];
  __shared__ float sf[kWaves];
  __shared__ unsigned long long sk[kWaves];
  const int64_t t = blockIdx.x;
  const typename T::raw* x = static_cast<const typename T::raw*>(a.logits) + t * a.ld;
  const int64_t V = a.vocab;
  float m = -kInf, bad = 0.f;
  for (int64_t v = threadIdx.x; v < V; v += kThreads) {
    const float f = T::widen(x[v]);
    m = fmaxf(m, f);
    if (!(f < kInf)) bad = 1.f;
  }
  m = block_reduce(m, sf, [](float p, float q) { return fmaxf(p, q); });
  bad = block_reduce(bad, sf, [](float p, float q) { return fmaxf(p, q); });
  double S = 0, E = 0;
  if (m > -kInf) {
    for (int64_t v = threadIdx.x; v < V; v += kThreads) {
      const float d = T::widen(x[v]) - m;
      const float e = expf(d);
      S += e;
      if (e > 0.f) E += double(e) * d;
    }
  }
  S = block_reduce(S, sd, [](double p, double q) { return p + q; });
  E = block_reduce(E, sd, [](double p, double q) { return p + q; });
  const bool empty = !(m > -kInf);
  const double logS = bad ? double(__builtin_nanf("")) : empty ? 0.0 : log(S);
  if (threadIdx.x == 0) {
    if (a.lse) a.lse[t] = float(double(m) + logS);
    if (a.entropy) a.entropy[t] = bad ? __builtin_nanf("") : empty ? 0.f : float(logS - E / S);
    if (a.logprob) {
      const int64_t tok = a.tokens[t];
      float lp = 0.f;
      if (tok >= V) lp = __builtin_nanf("");
      else if (tok >= 0) lp = empty && !bad ? -kInf : float(double(T::widen(x[tok])) - m - logS);
      a.logprob[t] = lp;
    }
  }
  unsigned long long last = ~0ull;
  for (int k = 0; k < a.top; ++k) {
    unsigned long long best = 0;
    if (!bad && last)
      for (int64_t v = threadIdx.x; v < V; v += kThreads) {
        const float f = T::widen(x[v]);
        const unsigned long long key = order_key(f, uint32_t(v));
        if (f > -kInf && key < last && key > best) best = key;
      }
    best = block_reduce(best, sk, [](unsigned long long p, unsigned long long q) { return p > q ? p : q; });
    if (threadIdx.x == 0) {
      a.top_token[t * a.top + k] = best ? int64_t(key_token(best)) : -1;
      a.top_logprob[t * a.top + k] =
          bad ? __builtin_nanf("") : best ? float(double(key_value(best)) - m - logS) : -kInf;
    }
    last = best;
  }
}

template <class T>
__global__ void __launch_bounds__(kThreads) logprobs_backward_kernel(LogprobGradArgs a) {
  const int64_t t = blockIdx.x, V = a.vocab;
  const typename T::raw* x = static_cast<const typename T::raw*>(a.logits) + t * a.ld;
  typename T::raw* out = static_cast<typename T::raw*>(a.grad) + t * a.ldg;
  const float lse = a.lse[t];
  const int64_t tok = a.tokens ? a.tokens[t] : -1;
  const float g = a.g && tok >= 0 ? a.g[t] : 0.f;
  const bool outside = a.g && tok >= V;
  const float h = a.h ? a.h[t] : 0.f, H = a.h ? a.entropy[t] : 0.f;
  const bool empty = lse == -kInf;
  for (int64_t v = int64_t(blockIdx.y) * kThreads + threadIdx.x; v < V;
       v += int64_t(gridDim.y) * kThreads) {
    const float xv = T::widen(x[v]);
    const float lp = xv - lse;
    const float p = expf(lp);
    float d = v == tok ? g : 0.f;
    if (p != 0.f) d -= p * fmaf(h, lp + H, g);   // a NaN counts as different from 0
    out[v] = T::narrow(outside ? __builtin_nanf("") : empty ? 0.f : d);
  }
}

}  // namespace

size_t token_logprobs_workspace_bytes(int64_t, int64_t, int) { return 0; }

hipError_t launch_token_logprobs(const LogprobArgs& a, int type, void*, hipStream_t stream) {
  return with_type(type, [&](auto t) {
    hipLaunchKernelGGL(logprobs_kernel<decltype(t)>, dim3(unsigned(a.nrows)), dim3(kThreads), 0,
                       stream, a);
    return hipGetLastError();
  });
}

hipError_t launch_token_logprobs_backward(const LogprobGradArgs& a, int type, hipStream_t stream) {
  const int64_t parts = std::min<int64_t>((a.vocab + 8 * kThreads - 1) / (8 * kThreads), 65535);
  return with_type(type, [&](auto t) {
    hipLaunchKernelGGL(logprobs_backward_kernel<decltype(t)>,
                       dim3(unsigned(a.nrows), unsigned(parts)), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
  });
}

}  // namespace seedq
