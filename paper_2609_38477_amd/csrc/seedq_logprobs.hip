// Log probabilities of given tokens with entropy and top alternatives, and their
// gradient at the logits.
//
// Both are one pass over the logits in 16-byte vectors, bound by memory. Forward, each
// thread keeps a running maximum m and, relative to it, S = sum e^(x - m) and
// E = sum e^(x - m) (x - m) in fp32; a larger maximum rescales both. The threads' sums meet
// in fp64, weighted by e^ of their maxima's distance in fp32, which errs by 2^-24 of the
// distance like every term. The entropy log S - E / S adds two terms of one sign.
#include <algorithm>
#include <cfloat>

#include "seedq_ops_device.h"

namespace seedq {
namespace {

typedef unsigned long long Key;

constexpr float kInf = __builtin_inff();
constexpr float kLog2E = 1.44269504088896340736f;
constexpr float kFar = -1e30f;      // stands in for x - m = -inf: its e^ is 0, and so is 0 x kFar
constexpr int kUnroll = 4;          // vectors in flight a thread
constexpr int kMaxTop = SEEDQ_MAX_TOP;
constexpr int kManyPicked = 2 * kMaxTop;
constexpr int kMaxSegs = 16;

// Order of alternatives in one number: the value's pattern made monotonic (-0 is
// 0), then the lower index first. 0 stands for none.
__device__ __forceinline__ Key order_key(float x, uint32_t index) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
  const uint32_t k = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (Key(k) << 32) | (0xFFFFFFFFu - index);
}
__device__ __forceinline__ float key_value(Key key) {
  const uint32_t k = uint32_t(key >> 32);
  return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ uint32_t key_index(Key key) { return 0xFFFFFFFFu - uint32_t(key); }
__device__ __forceinline__ Key max_key(Key a, Key b) { return a > b ? a : b; }

// A row in 16-byte vectors and the elements after the last.
template <class T>
struct Row {
  static constexpr int N = kPerVector<T>;
  const typename T::raw* x;
  uint32_t vectors, tail;   // a row has fewer than 2^31 elements
  __device__ Row(const typename T::raw* p, int64_t n)
      : x(p), vectors(uint32_t(n) / N), tail(uint32_t(n) % N) {}
  __device__ __forceinline__ uint32x4 load(uint32_t i) const { return load16(x + size_t(i) * N); }
};

template <class T>
__device__ __forceinline__ uint32x4 minus_infinity() {
  const uint32_t w = kPerVector<T> == 4 ? 0xFF800000u : uint32_t(T::narrow(-kInf)) * 0x10001u;
  return uint32x4{w, w, w, w};
}

struct Sums {
  float m = -FLT_MAX, S = 0.f, E = 0.f;
  float best = -kInf;       // the largest element seen and the first vector that has it
  uint32_t base = 0;

  __device__ __forceinline__ void raise(float to) {
    if (to > m) {
      const float d = fmaxf(m - to, kFar);
      const float c = __builtin_amdgcn_exp2f(d * kLog2E);
      E = c * fmaf(d, S, E);
      S *= c;
      m = to;
    }
  }
  __device__ __forceinline__ void add(float x) {
    // a NaN stays one: m is infinite only in a row without a distribution
    const float d = __builtin_elementwise_maximum(x - m, kFar);
    const float e = __builtin_amdgcn_exp2f(d * kLog2E);
    S += e;
    E = fmaf(e, d, E);
  }
  __device__ __forceinline__ void note(float largest, uint32_t at) {
    if (largest > best) {
      best = largest;
      base = at;
    }
  }
};

template <int N>
__device__ __forceinline__ float largest(const float (&f)[N]) {
  float t = f[0];
#pragma unroll
  for (int i = 1; i < N; ++i) t = fmaxf(t, f[i]);
  return t;
}

// What a segment of a row hands to the join.
struct Partial {
  double S, E;
  float m, unused;
};

// The logit of a row's token. It is asked for before the sums meet, so that it is there
// when they have.
template <class T>
__device__ __forceinline__ float token_logit(const LogprobArgs& a, int64_t t, int64_t tok) {
  const typename T::raw* x = static_cast<const typename T::raw*>(a.logits) + t * a.ld;
  return T::widen(x[tok >= 0 && tok < a.vocab ? tok : 0]);
}

// log S; S is 0 in a row without a finite logit and NaN in one without a distribution.
__device__ __forceinline__ double log_of(double S) { return S == 0.0 ? -double(kInf) : log(S); }

// The outputs of row t but for the alternatives, by one thread.
__device__ __forceinline__ void write_sums(const LogprobArgs& a, int64_t t, int64_t tok, float x,
                                           float m, double S, double E, double log_s) {
  const bool empty = S == 0.0;
  if (a.lse) a.lse[t] = empty ? -kInf : float(double(m) + log_s);
  if (a.entropy) a.entropy[t] = empty ? 0.f : float(log_s - E / S);
  if (a.logprob) {
    const double lp = empty ? -double(kInf) : (double(x) - m) - log_s;
    a.logprob[t] = tok < 0 ? 0.f : tok >= a.vocab ? __builtin_nanf("") : float(lp);
  }
}

__device__ __forceinline__ void write_alternative(const LogprobArgs& a, int64_t t, int k, Key key,
                                                  float m, double log_s) {
  const bool bad = !(log_s <= double(FLT_MAX));   // NaN
  const bool none = bad || key == 0;
  a.top_token[t * a.top + k] = none ? -1 : int64_t(key_index(key));
  a.top_logprob[t * a.top + k] =
      bad ? __builtin_nanf("") : none ? -kInf : float((double(key_value(key)) - m) - log_s);
}

// The keys of list[0 .. n) in falling order: f(rank, key) for the first `top` ranks.
template <class F>
__device__ __forceinline__ void by_rank(const Key* list, int n, int top, F f) {
  for (int i = int(threadIdx.x); i < n; i += int(blockDim.x)) {
    const Key mine = list[i];
    int rank = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) rank += list[j] > mine ? 1 : 0;
    if (rank < top) f(rank, mine);
  }
}

// One workgroup of NT threads a row, or a segment of one (blockIdx.y of segs), whose
// sums and alternatives then go to the join.
//
// Alternatives: a thread remembers its largest element and the vector that first had it.
// The top-th largest of the largest keys of 64 groups of threads bounds the top-th
// largest element from below (where many keys reach it, as among equal logits, the
// top-th largest key takes its place), so only the vectors of threads whose keys reach
// the bound are read again, by all threads together, and the elements that reach it are
// ranked against each other. Vectors are intervals of the row, so the order of (value,
// first vector) is that of (value, index), and ties are cut the same way. A thread's
// vectors lie in as many cache lines, which is what the second look costs: 2048 rows of
// 131072 bf16 logits take 109 us with 5 alternatives, 118 with 20 and 110 with none. For
// few rows the launch spends its time on the way through the code, so that is kept short:
// one row of 32000 fp32 logits takes 5.7 us without alternatives and 8.7 with 20.
template <class T, int NT>
__global__ void __launch_bounds__(NT)
logprobs_kernel(LogprobArgs a, uint32_t segs, uint32_t seg_vectors,
                Partial* __restrict__ partial, Key* __restrict__ seg_top) {
  constexpr int N = kPerVector<T>, kWaves = NT / 64, kGroup = NT / 64;
  constexpr int kPicked = kMaxTop * kGroup;        // the keys of kMaxTop groups
  constexpr int kFound = NT == 64 ? 512 : 1024;    // elements kept before the slow selection
  __shared__ double sd[2][kWaves];
  __shared__ float sf[kWaves];
  __shared__ Key group_key[64], picked[kPicked], found[kFound], tighter;
  __shared__ int npicked, nfound;
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, seg = blockIdx.y;
  const int64_t t = blockIdx.x;
  const Row<T> row(static_cast<const typename T::raw*>(a.logits) + t * a.ld, a.vocab);
  const int64_t tok = a.tokens ? a.tokens[t] : -1;
  const uint32_t begin = std::min(seg * seg_vectors, row.vectors);
  const uint32_t end = std::min(begin + seg_vectors, row.vectors);
  Sums s;
#pragma unroll 1
  for (uint32_t i = begin; i < end; i += kUnroll * NT) {
    uint32x4 v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      v[u] = minus_infinity<T>();   // adds nothing
      if (i + u * NT + tid < end) v[u] = row.load(i + u * NT + tid);
    }
    float f[kUnroll][N], top = -kInf;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      widen<T>(v[u], f[u]);
      const float l = largest(f[u]);
      s.note(l, (i + u * NT + tid) * N);
      top = fmaxf(top, l);
    }
    s.raise(top);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (i + u * NT < end)
#pragma unroll
        for (int k = 0; k < N; ++k) s.add(f[u][k]);
  }
  const uint32_t after = row.vectors * N;
  const bool has_tail = seg == segs - 1 && tid < row.tail;   // elements after the last vector
  if (has_tail) {
    const float x = T::widen(row.x[after + tid]);
    s.raise(x);
    s.add(x);
    s.note(x, after + tid);
  }
  const Key mine = s.best > -kInf ? order_key(s.best, s.base) : 0;

  const float xtok = segs == 1 ? token_logit<T>(a, t, tok) : 0.f;
  // the sums of the threads
  float m = lanes_reduce(s.m, [](float p, float q) { return fmaxf(p, q); });
  if (lane == 0) sf[wave] = m;
  if (tid == 0) npicked = nfound = 0;
  __syncthreads();
  m = sf[0];
  for (int w = 1; w < kWaves; ++w) m = fmaxf(m, sf[w]);
  const float d = fmaxf(s.m - m, kFar);
  const double c = __builtin_amdgcn_exp2f(d * kLog2E);
  const auto add = [](double p, double q) { return p + q; };
  double S = lanes_reduce(c * s.S, add), E = lanes_reduce(c * (s.E + double(d) * s.S), add);
  if (lane == 0) {
    sd[0][wave] = S;
    sd[1][wave] = E;
  }
  // the largest element of each of 64 groups of threads
  const Key g = lanes_reduce<kGroup>(mine, max_key);
  if (tid % kGroup == 0) group_key[tid / kGroup] = g;
  __syncthreads();
  S = sd[0][0], E = sd[1][0];
  for (int w = 1; w < kWaves; ++w) {
    S += sd[0][w];
    E += sd[1][w];
  }
  const double log_s = log_of(S);
  const int64_t at = t * int64_t(segs) + seg;
  if (tid == 0) {
    if (segs > 1) partial[at] = Partial{S, E, m, 0.f};
    else write_sums(a, t, tok, xtok, m, S, E, log_s);
  }
  if (a.top == 0) return;
  auto put = [&](int rank, Key key) {
    if (segs > 1) seg_top[at * a.top + rank] = key;
    else write_alternative(a, t, rank, key, m, log_s);
  };
  if (!(S > 0.0)) {   // nothing left, or no distribution (the same for all threads)
    for (int k = int(tid); k < a.top; k += NT) put(k, 0);
    return;
  }
  Key bound;
  {   // every wave for itself
    const Key key = group_key[lane];
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < 64; ++j) rank += group_key[j] > key ? 1 : 0;
    const unsigned long long cut = __ballot(rank == a.top - 1);
    bound = cut ? max_key(__shfl(key, __builtin_ctzll(cut), 64), 1) : 1;   // fewer groups: all keys
    if (mine >= bound) picked[atomicAdd(&npicked, 1)] = mine;
  }
  __syncthreads();
  const int npick = npicked;
  if (npick > kManyPicked) {
    by_rank(picked, npick, a.top, [&](int rank, Key key) {
      if (rank == a.top - 1) tighter = key;
    });
    __syncthreads();
    bound = tighter;
  }
  auto take = [&](float x, uint32_t index, uint32_t base) {
    if (x > -kInf && order_key(x, base) >= bound) {
      const int k = atomicAdd(&nfound, 1);
      if (k < kFound) found[k] = order_key(x, index);
    }
  };
  // all threads over (picked key, the vectors of its thread)
  const uint32_t each = (end - begin + NT - 1) / NT;
#pragma unroll 1
  for (uint32_t p = tid; p < uint32_t(npick) * each; p += NT) {
    const uint32_t which = p / each;
    const Key key = picked[which];
    const uint32_t e = key_index(key);
    const uint32_t owner = e < after ? (e / N - begin) % NT : e - after;
    const uint32_t v = begin + owner + (p - which * each) * NT;
    if (key < bound || v >= end) continue;
    float f[N];
    widen<T>(row.load(v), f);
    if (order_key(largest(f), v * N) >= bound)
#pragma unroll
      for (int k = 0; k < N; ++k) take(f[k], v * N + k, v * N);
  }
  if (has_tail) take(T::widen(row.x[after + tid]), after + tid, after + tid);
  __syncthreads();
  const int n = nfound;
  if (n <= kFound) {
    by_rank(found, n, a.top, put);
    for (int k = n + int(tid); k < a.top; k += NT) put(k, 0);
    return;
  }
  // More elements reach the bound than are kept, as when a thread's elements are all
  // among the largest: one pass over the segment for each alternative.
  Key last = ~Key(0);
  const uint32_t stop = seg == segs - 1 ? uint32_t(a.vocab) : end * N;
#pragma unroll 1
  for (int k = 0; k < a.top; ++k) {
    Key best = 0;
#pragma unroll 1
    for (uint32_t e = begin * N + tid; e < stop; e += NT) {
      const float x = T::widen(row.x[e]);
      const Key key = order_key(x, e);
      if (x > -kInf && key < last && key > best) best = key;
    }
    best = lanes_reduce(best, max_key);
    __syncthreads();
    if (lane == 0) picked[wave] = best;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) best = max_key(best, picked[w]);
    if (tid == 0) put(k, best);
    last = best ? best : 1;   // after the last one nothing is below
  }
}

// The segments of a row: sums in the order of the segments, alternatives of all of them
// ranked against each other.
template <class T>
__global__ void __launch_bounds__(256) logprobs_join_kernel(LogprobArgs a, int segs,
                                                            const Partial* __restrict__ partial,
                                                            const Key* __restrict__ seg_top) {
  __shared__ Key keys[kMaxSegs * kMaxTop];
  __shared__ int n;
  const int64_t t = blockIdx.x;
  const Partial* part = partial + t * segs;
  const int64_t tok = a.tokens ? a.tokens[t] : -1;
  const float xtok = token_logit<T>(a, t, tok);
  float m = part[0].m;
  for (int s = 1; s < segs; ++s) m = fmaxf(m, part[s].m);
  double S = 0, E = 0;
  for (int s = 0; s < segs; ++s) {
    const float d = fmaxf(part[s].m - m, kFar);
    const double c = __builtin_amdgcn_exp2f(d * kLog2E);
    S += c * part[s].S;
    E += c * (part[s].E + double(d) * part[s].S);
  }
  const double log_s = log_of(S);
  if (threadIdx.x == 0) {
    write_sums(a, t, tok, xtok, m, S, E, log_s);
    n = 0;
  }
  if (a.top == 0) return;
  __syncthreads();
  // no segment's last alternative is beaten by fewer than `top`
  const Key* in = seg_top + t * segs * a.top;
  Key bound = 1;
  for (int s = 0; s < segs; ++s) bound = max_key(bound, in[s * a.top + a.top - 1]);
  for (int k = int(threadIdx.x); k < segs * a.top; k += 256)
    if (in[k] >= bound) keys[atomicAdd(&n, 1)] = in[k];
  __syncthreads();
  const int count = S > 0.0 ? n : 0;
  by_rank(keys, count, a.top, [&](int rank, Key key) { write_alternative(a, t, rank, key, m, log_s); });
  for (int k = count + int(threadIdx.x); k < a.top; k += 256) write_alternative(a, t, k, 0, m, log_s);
}

// ---------------------------------------------------------------- gradient

constexpr int kGradThreads = 256;
// An lse in fp32 errs by 2^-24 of itself, and e^(x - lse) by as much of 1: from here on by
// 2^-14 and more, all of it in a row of the type's lowest value. Such a row's p are taken
// from its own largest logit and sum.
constexpr float kFarLse = 1024.f;

// The largest logit of a row and the log of its sum relative to it, for all threads, by one
// workgroup that has read the whole row when this returns.
template <class T>
__device__ __forceinline__ void largest_and_log_sum(const Row<T>& row, float& m, float& log_s) {
  constexpr int kWaves = kGradThreads / 64;
  __shared__ float sm[kWaves];
  __shared__ double ss[kWaves];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  Sums s;
#pragma unroll 1
  for (uint32_t i = tid; i < row.vectors; i += kGradThreads) {
    float f[kPerVector<T>];
    widen<T>(row.load(i), f);
    s.raise(largest(f));
#pragma unroll
    for (int k = 0; k < kPerVector<T>; ++k) s.add(f[k]);
  }
  if (tid < row.tail) {
    const float x = T::widen(row.x[row.vectors * kPerVector<T> + tid]);
    s.raise(x);
    s.add(x);
  }
  m = lanes_reduce(s.m, [](float p, float q) { return fmaxf(p, q); });
  if (lane == 0) sm[wave] = m;
  __syncthreads();
  m = sm[0];
  for (int w = 1; w < kWaves; ++w) m = fmaxf(m, sm[w]);
  const double c = __builtin_amdgcn_exp2f(fmaxf(s.m - m, kFar) * kLog2E);
  double S = lanes_reduce(c * s.S, [](double p, double q) { return p + q; });
  if (lane == 0) ss[wave] = S;
  __syncthreads();
  S = ss[0];
  for (int w = 1; w < kWaves; ++w) S += ss[w];
  log_s = float(log(S));
}

struct GradRow {
  float lse, g, h, H;
  float m = 0.f, log_s = 0.f;   // lse in two parts, in a far row
  int64_t tok;
  bool empty, outside, far;
  __device__ GradRow(const LogprobGradArgs& a, int64_t t) {
    lse = a.lse[t];
    tok = a.tokens ? a.tokens[t] : -1;
    g = a.g && tok >= 0 ? a.g[t] : 0.f;
    outside = a.g && tok >= a.vocab;
    h = a.h ? a.h[t] : 0.f;
    H = a.h ? a.entropy[t] : 0.f;
    empty = lse == -kInf;
    far = fabsf(lse) >= kFarLse && fabsf(lse) < kInf;
  }
  template <bool FAR>
  __device__ __forceinline__ float at(float x, int64_t v) const {
    const float lp = FAR ? (x - m) - log_s : x - lse;
    const float p = __builtin_amdgcn_exp2f(lp * kLog2E);
    float d = v == tok ? g : 0.f;
    if (p != 0.f) d -= p * fmaf(h, lp + H, g);   // a NaN counts as different from 0
    return outside ? __builtin_nanf("") : empty ? 0.f : d;
  }
};

// The gradients of a row's vectors from `first` on, kUnroll a thread and step of `by`
// vectors, and of the elements after the last vector.
template <class T, bool FAR>
__device__ __forceinline__ void write_gradient(const Row<T>& row, const GradRow& r,
                                               typename T::raw* out, int64_t first, int64_t by) {
  constexpr int N = kPerVector<T>;
  const uint32_t tid = threadIdx.x;
  if (first == 0 && tid < row.tail) {
    const uint32_t e = row.vectors * N + tid;
    out[e] = T::narrow(r.template at<FAR>(T::widen(row.x[e]), e));
  }
  for (int64_t b = first; b < row.vectors; b += by) {
    uint32x4 v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t i = b + u * kGradThreads + tid;
      if (i < row.vectors) v[u] = row.load(uint32_t(i));
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t i = b + u * kGradThreads + tid;
      if (i >= row.vectors) break;
      float f[N];
      widen<T>(v[u], f);
#pragma unroll
      for (int k = 0; k < N; ++k) f[k] = r.template at<FAR>(f[k], i * N + k);
      store16(out + i * N, narrow<T>(f));
    }
  }
}

// The workgroups of a row (blockIdx.y) take kUnroll vectors a thread of it in turn. A far
// row is the first one's alone, which reads it twice: the gradient may lie on the logits.
// 4096 x 32000 bf16 takes 110 us, with far rows only 141, in fp32 212 and 297; a single far
// row of 131072 59 us, where an ordinary one takes 3.3.
template <class T>
__global__ void __launch_bounds__(kGradThreads) logprobs_backward_kernel(LogprobGradArgs a) {
  constexpr int64_t kStep = int64_t(kUnroll) * kGradThreads;
  const int64_t t = blockIdx.x;
  const Row<T> row(static_cast<const typename T::raw*>(a.logits) + t * a.ld, a.vocab);
  typename T::raw* out = static_cast<typename T::raw*>(a.grad) + t * a.ldg;
  GradRow r(a, t);
  if (r.far) {
    if (blockIdx.y != 0) return;
    largest_and_log_sum<T>(row, r.m, r.log_s);
    write_gradient<T, true>(row, r, out, 0, kStep);
  } else {
    write_gradient<T, false>(row, r, out, int64_t(blockIdx.y) * kStep, int64_t(gridDim.y) * kStep);
  }
}

size_t partial_bytes(int64_t nrows, int segs) {
  return align256(size_t(nrows) * segs * sizeof(Partial));
}

// Segments of a row: with few rows, rows of 2^18 bytes and more are cut so that a
// workgroup has 8 vectors a thread, up to a workgroup for each CU. The join is a second
// kernel, so shorter rows are left whole: 1 x 64000 fp32 with 20 alternatives takes 12.1
// us whole and 13.1 in four, 1 x 131072 fp32 with 5 16.6 and 12.7 in eight, 64 x 131072
// bf16 17.6 and 15.2 in four, 128 x 60000 fp32 13.2 and 16.7 in four.
int segments(int64_t nrows, int64_t vocab, int per_vector) {
  const int64_t n = vocab / per_vector;
  if (n < 16384) return 1;
  return int(std::max<int64_t>(1, std::min<int64_t>({n / 4096, 256 / nrows, kMaxSegs})));
}

}  // namespace

// Bytes for up to kMaxRows rows.
static size_t rows_bytes(int64_t nrows, int64_t vocab, int top) {
  const int segs = segments(nrows, vocab, 4);   // the type with the most
  if (segs == 1) return 0;
  return partial_bytes(nrows, segs) + align256(size_t(nrows) * segs * top * sizeof(Key));
}

size_t token_logprobs_workspace_bytes(int64_t nrows, int64_t vocab, int top) {
  size_t need = rows_bytes(std::min(nrows, kMaxRows), vocab, top);
  // the last launch of many may have few rows and cut them
  if (nrows > kMaxRows && nrows % kMaxRows)
    need = std::max(need, rows_bytes(nrows % kMaxRows, vocab, top));
  return need;
}

hipError_t launch_token_logprobs(const LogprobArgs& all, int type, void* d_ws, hipStream_t stream) {
  if (all.nrows > kMaxRows) {   // the launches follow each other and share the workspace
    for (int64_t r = 0; r < all.nrows; r += kMaxRows) {
      const auto from = [&](auto* p, int64_t each) { return p ? p + r * each : p; };
      LogprobArgs a = all;
      a.logits = static_cast<const char*>(all.logits) + r * all.ld * (type == SEEDQ_F32 ? 4 : 2);
      a.nrows = std::min(kMaxRows, all.nrows - r);
      a.tokens = from(all.tokens, 1);
      a.logprob = from(all.logprob, 1), a.entropy = from(all.entropy, 1), a.lse = from(all.lse, 1);
      a.top_token = from(all.top_token, all.top), a.top_logprob = from(all.top_logprob, all.top);
      const hipError_t e = launch_token_logprobs(a, type, d_ws, stream);
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    const LogprobArgs& a = all;
    const int segs = segments(a.nrows, a.vocab, kPerVector<T>);
    Partial* part = static_cast<Partial*>(d_ws);
    Key* keys = reinterpret_cast<Key*>(static_cast<char*>(d_ws) + partial_bytes(a.nrows, segs));
    const uint32_t n = uint32_t(a.vocab) / kPerVector<T>;
    auto go = [&](auto kern, unsigned threads) {
      hipLaunchKernelGGL(kern, dim3(unsigned(a.nrows), unsigned(segs)), dim3(threads), 0, stream, a,
                         uint32_t(segs), (n + segs - 1) / segs, part, keys);
    };
    // One wave where a row is short, or rather short and there are many (4096 x 4000 bf16
    // 15.0 us, with 4 waves 22.1; 700 x 16000 16.6 and 12.1); eight where it is long or
    // there are few (2048 x 131072 bf16 109 us, with 4 waves 111; 1 x 32000 fp32 9.0 and
    // 12.1; 4096 x 32000 bf16 66 and 62).
    if (n <= 256 || (n <= 1024 && a.nrows >= 1024)) go(logprobs_kernel<T, 64>, 64);
    else if (n < 8192 && a.nrows > 512) go(logprobs_kernel<T, 256>, 256);
    else go(logprobs_kernel<T, 512>, 512);
    if (segs > 1)
      hipLaunchKernelGGL(logprobs_join_kernel<T>, dim3(unsigned(a.nrows)), dim3(256), 0, stream, a,
                         segs, part, keys);
    return hipGetLastError();
  });
}

hipError_t launch_token_logprobs_backward(const LogprobGradArgs& all, int type, hipStream_t stream) {
  if (all.nrows > kMaxRows) {
    for (int64_t r = 0; r < all.nrows; r += kMaxRows) {
      const auto from = [&](auto* p) { return p ? p + r : p; };
      const int64_t size = type == SEEDQ_F32 ? 4 : 2;
      LogprobGradArgs a = all;
      a.logits = static_cast<const char*>(all.logits) + r * all.ld * size;
      a.grad = static_cast<char*>(all.grad) + r * all.ldg * size;
      a.nrows = std::min(kMaxRows, all.nrows - r);
      a.tokens = from(all.tokens);
      a.lse = from(all.lse), a.entropy = from(all.entropy), a.g = from(all.g), a.h = from(all.h);
      const hipError_t e = launch_token_logprobs_backward(a, type, stream);
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    const LogprobGradArgs& a = all;
    const int64_t step = int64_t(kUnroll) * kGradThreads * kPerVector<T>;
    const dim3 grid(unsigned(a.nrows),
                    unsigned(std::min<int64_t>((a.vocab + step - 1) / step, 65535)));
    hipLaunchKernelGGL(logprobs_backward_kernel<T>, grid, dim3(kGradThreads), 0, stream, a);
    return hipGetLastError();
  });
}

}  // namespace seedq
