// The largest elements of a row of logits in the order of (value, lower index), by one
// workgroup that goes over the row once.
//
// A thread remembers its largest element and the vector that first had it. The top-th
// largest of the largest keys of 64 groups of threads bounds the top-th largest element
// from below (where many keys reach it, as among equal logits, the top-th largest key
// takes its place), so only the vectors of threads whose keys reach the bound are read
// again, by all threads together, and the elements that reach it are ranked against each
// other. Vectors are intervals of the row, so the order of (value, first vector) is that
// of (value, index), and ties are cut the same way.
#pragma once

#include <algorithm>

#include "seedq_ops_device.h"

namespace seedq {

typedef unsigned long long Key;

constexpr float kInf = __builtin_inff();
constexpr int kMaxTop = SEEDQ_MAX_TOP;
constexpr int kManyPicked = 2 * kMaxTop;

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

template <int N>
__device__ __forceinline__ float largest(const float (&f)[N]) {
  float t = f[0];
#pragma unroll
  for (int i = 1; i < N; ++i) t = fmaxf(t, f[i]);
  return t;
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

// What the selection keeps in LDS.
template <int NT>
struct Chosen {
  static constexpr int kGroup = NT / 64;
  static constexpr int kPicked = kMaxTop * kGroup;        // the keys of kMaxTop groups
  static constexpr int kFound = NT == 64 ? 512 : 1024;    // elements kept before the slow selection
  Key group_key[64], picked[kPicked], found[kFound], tighter;
  int npicked, nfound;   // 0 before top_finish, by the caller
};

// The largest element of each of 64 groups of threads. mine: the thread's largest element
// and the vector that first had it, 0 for none. A barrier follows.
template <int NT>
__device__ __forceinline__ void top_note(Chosen<NT>& c, Key mine) {
  const Key g = lanes_reduce<NT / 64>(mine, max_key);
  if (threadIdx.x % (NT / 64) == 0) c.group_key[threadIdx.x / (NT / 64)] = g;
}

// put(rank, key) for the `top` largest elements of the row's vectors begin .. end, which
// thread i took i, i + NT, ... of, and, in the last segment, of what lies after the last
// vector (has_tail: this thread had one of those).
template <class T, int NT, class Put>
__device__ __forceinline__ void top_finish(Chosen<NT>& c, const Row<T>& row, uint32_t begin, uint32_t end,
                                           bool has_tail, bool last_segment, Key mine, int top, Put put) {
  constexpr int N = kPerVector<T>, kWaves = NT / 64;
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t after = row.vectors * N;
  Key bound;
  {   // every wave for itself
    const Key key = c.group_key[lane];
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < 64; ++j) rank += c.group_key[j] > key ? 1 : 0;
    const unsigned long long cut = __ballot(rank == top - 1);
    bound = cut ? max_key(__shfl(key, __builtin_ctzll(cut), 64), 1) : 1;   // fewer groups: all keys
    if (mine >= bound) c.picked[atomicAdd(&c.npicked, 1)] = mine;
  }
  __syncthreads();
  const int npick = c.npicked;
  if (npick > kManyPicked) {
    by_rank(c.picked, npick, top, [&](int rank, Key key) {
      if (rank == top - 1) c.tighter = key;
    });
    __syncthreads();
    bound = c.tighter;
  }
  auto take = [&](float x, uint32_t index, uint32_t base) {
    if (x > -kInf && order_key(x, base) >= bound) {
      const int k = atomicAdd(&c.nfound, 1);
      if (k < Chosen<NT>::kFound) c.found[k] = order_key(x, index);
    }
  };
  // all threads over (picked key, the vectors of its thread)
  const uint32_t each = (end - begin + NT - 1) / NT;
#pragma unroll 1
  for (uint32_t p = tid; p < uint32_t(npick) * each; p += NT) {
    const uint32_t which = p / each;
    const Key key = c.picked[which];
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
  const int n = c.nfound;
  if (n <= Chosen<NT>::kFound) {
    by_rank(c.found, n, top, put);
    for (int k = n + int(tid); k < top; k += NT) put(k, 0);
    return;
  }
  // More elements reach the bound than are kept, as when a thread's elements are all
  // among the largest: one pass over the segment for each alternative.
  Key last = ~Key(0);
  const uint32_t stop = last_segment ? row.vectors * N + row.tail : end * N;
#pragma unroll 1
  for (int k = 0; k < top; ++k) {
    Key best = 0;
#pragma unroll 1
    for (uint32_t e = begin * N + tid; e < stop; e += NT) {
      const float x = T::widen(row.x[e]);
      const Key key = order_key(x, e);
      if (x > -kInf && key < last && key > best) best = key;
    }
    best = lanes_reduce(best, max_key);
    __syncthreads();
    if (lane == 0) c.picked[wave] = best;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) best = max_key(best, c.picked[w]);
    if (tid == 0) put(k, best);
    last = best ? best : 1;   // after the last one nothing is below
  }
}

}  // namespace seedq
