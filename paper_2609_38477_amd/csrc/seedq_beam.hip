// One step of beam search: the selection over beams and vocabulary, and the states of the
// beams moved to those that continue them.
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "seedq_beam_internal.h"
#include "seedq_top.h"

namespace seedq {
namespace {

constexpr double kLog2EExact = 1.44269504088896340736, kLn2 = 0.693147180559945309417;
constexpr float kLog2E = float(kLog2EExact), kLog2E16 = 0x1.7154p0f, kLn2High = float(kLn2), kLn2Low = float(kLn2 - double(kLn2High));
constexpr int kUnroll = 4;          // vectors in flight a thread
constexpr int kMaxSegs = 16;
constexpr int kMaxBeams = SEEDQ_MAX_BEAMS;
static_assert(SEEDQ_MAX_BEAM_TOP <= kMaxTop, "the selection of a row");

// ---------------------------------------------------------------- selection
//
// total(b, v) = s_b + (x_bv - log sum e^x_b). Within a beam the order is that of the logits, so no
// more than the `top` largest of each row can be among a sequence's: the first kernel goes over
// the logits once and leaves of every row, or segment of one, its sum of exponentials and the
// keys of its largest elements, the second ranks what the beams of a sequence offer.
//
// Totals of different beams may lie next to each other, and where many tokens lie as far below
// the largest as each other, what one term errs by the sum errs by. So a term is rounded in the
// exponential alone, by 8.5e-8 of itself at the most (the instruction over all arguments); what
// its argument was rounded by is added to the sum. Pairs (6e-8) are joined in fp64. The sum errs
// by less than 1.75e-7 of itself, 2.8e-8 of them the square of a bfloat16 argument's rest, next to
// +-48. Exponentials of fp32 differences and sums of 32 of them took 6.4e-7, for 131072 equal
// logits 11 below the largest.
//
// Memory bounds the first: 512 rows of 131072 bf16 logits take 29 to 31 us (4.3 to 4.6 TB/s); 4 rows
// of 32003 fp32 7, latency. The second takes 7 us for 64 sequences of 8 beams, 6 for one, its
// way from load to load (13 and 9 where it read keys when it needed them).

// A sum stands for e^at times as much, at being 0 for a largest element of less than 48 either way,
// so that its terms are powers of the logits themselves, and else that element: fp32 then holds the
// differences to all that count.
__device__ __forceinline__ float scale_of(float m) { return fabsf(m) < 48.f ? 0.f : m; }
__device__ __forceinline__ double rescaled(double S, float from, float to) {
  if (from == to || S == 0.0) return S;
  return S * exp2((double(from) - double(to)) * kLog2EExact);
}

struct Partial {
  double S;
  float m, unused;
};

__device__ __forceinline__ bool offers_tokens(const BeamArgs& a, int64_t t) {
  return !(a.finished && a.finished[t]) && a.scores[t] != -kInf;
}

// One workgroup of NT threads a row, or a segment of one (blockIdx.y of segs).
template <class T, int NT>
__global__ void __launch_bounds__(NT)
beam_rows_kernel(BeamArgs a, uint32_t segs, uint32_t seg_vectors, Partial* __restrict__ partial,
                 Key* __restrict__ seg_top) {
  constexpr int N = kPerVector<T>, kWaves = NT / 64;
  __shared__ double sd[kWaves];
  __shared__ float sf[kWaves];
  __shared__ Chosen<NT> chosen;
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, seg = blockIdx.y;
  const int64_t t = blockIdx.x;
  if (!offers_tokens(a, t)) return;
  const Row<T> row(static_cast<const typename T::raw*>(a.logits) + t * a.ld, a.vocab);
  const uint32_t begin = std::min(seg * seg_vectors, row.vectors);
  const uint32_t end = std::min(begin + seg_vectors, row.vectors);
  float m = -FLT_MAX, best = -kInf;
  float scale = m;
  double S = 0.0;
  uint32_t base = 0;
  const auto raise = [&](float to) {
    if (to > m) {
      m = to;
      S = rescaled(S, scale, scale_of(m));
      scale = scale_of(m);
    }
  };
  // The terms of all vectors. e^c = 2^p e^(c - p log 2), of which the second factor less 1, times the
  // first, is added up apart. p is c log2 e, and of a bfloat16 the product with the first 16 bits of
  // log2 e, which is exact. A NaN stays one and +inf becomes one; -inf is 0.
  const auto add = [&](const float (&f)[N], float& rest, auto whole) {
    constexpr bool kScaled = !decltype(whole)::value, kExact = !kScaled && std::is_same_v<T, BF16>;
    const auto term = [&](float x) {
      const float c = __builtin_elementwise_maximum(kScaled ? x - scale : x, -104.f);
      const float p = c * (kExact ? kLog2E16 : kLog2E), e = __builtin_amdgcn_exp2f(p);
      rest = fmaf(e, kExact ? c : fmaf(p, -kLn2Low, fmaf(p, -kLn2High, c)), rest);
      return e;
    };
#pragma unroll
    for (int k = 0; k < N; k += 2) {
      const float a = term(f[k]);
      S += double(a + term(f[k + 1]));
    }
  };
  const auto note = [&](float l, uint32_t at) {
    if (l > best) {
      best = l;
      base = at;
    }
  };
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
      note(l, (i + u * NT + tid) * N);
      top = fmaxf(top, l);
    }
    raise(top);
    const auto all = [&](auto whole) {
      float rest = 0.f;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (i + u * NT < end) add(f[u], rest, whole);
      S += double(rest) * (decltype(whole)::value && std::is_same_v<T, BF16> ? 1.0 - double(kLog2E16) * kLn2 : 1.0);
    };
    if (__any(scale != 0.f)) all(std::false_type{});
    else all(std::true_type{});
  }
  const uint32_t after = row.vectors * N;
  const bool has_tail = seg == segs - 1 && tid < row.tail;   // elements after the last vector
  if (has_tail) {
    const float x = T::widen(row.x[after + tid]);
    raise(x);
    S += exp(double(x) - double(scale));
    note(x, after + tid);
  }
  const Key mine = best > -kInf ? order_key(best, base) : 0;
  // the sums of the threads
  float most = lanes_reduce(m, [](float p, float q) { return fmaxf(p, q); });
  if (lane == 0) sf[wave] = most;
  if (tid == 0) chosen.npicked = chosen.nfound = 0;
  __syncthreads();
  most = sf[0];
  for (int w = 1; w < kWaves; ++w) most = fmaxf(most, sf[w]);
  S = rescaled(S, scale, scale_of(most));
  S = lanes_reduce(S, [](double p, double q) { return p + q; });
  if (lane == 0) sd[wave] = S;
  top_note<NT>(chosen, mine);
  __syncthreads();
  S = sd[0];
  for (int w = 1; w < kWaves; ++w) S += sd[w];
  const int64_t at = t * int64_t(segs) + seg;
  if (tid == 0) partial[at] = Partial{S, most, 0.f};
  auto put = [&](int rank, Key key) { seg_top[at * a.top + rank] = key; };
  if (!(S > 0.0)) {   // nothing left, or no distribution (the same for all threads)
    for (int k = int(tid); k < a.top; k += NT) put(k, 0);
    return;
  }
  top_finish<T, NT>(chosen, row, begin, end, has_tail, seg == segs - 1, mine, a.top, put);
}

// What a sequence may be continued by, in falling order: (total, beam, key) as two numbers.
struct Offer {
  uint64_t total;   // monotone in the total; 0 for none
  uint32_t beam;
  Key key;
  __device__ __forceinline__ bool before(const Offer& o) const {
    return (total > o.total) |
           ((total == o.total) & ((beam < o.beam) | ((beam == o.beam) & (key > o.key))));
  }
};
__device__ __forceinline__ uint64_t order_of(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v + 0.0);   // -0 is 0
  return b >> 63 ? ~b : b | uint64_t(1) << 63;
}
__device__ __forceinline__ double total_of(uint64_t k) {
  return __builtin_bit_cast(double, k >> 63 ? k & ~(uint64_t(1) << 63) : ~k);
}

// A workgroup a sequence. Its beams' segments are lists of offers in falling order. With as
// many lists as continuations the top-th best of their first offers bounds what is ranked;
// with fewer, the best of their last ones, or the worst of those so far down that there are
// `top` in all.
constexpr int kJoinThreads = 256;
constexpr int kMaxLists = kMaxBeams * kMaxSegs;
constexpr int kAhead = 2;    // keys of a thread that are read at once
__global__ void __launch_bounds__(kJoinThreads)
beam_join_kernel(BeamArgs a, int segs, const Partial* __restrict__ partial,
                 const Key* __restrict__ seg_top) {
  enum { kNone, kTokens, kFinished, kBad };
  __shared__ double most[kMaxBeams], log_s[kMaxBeams];
  __shared__ float score[kMaxBeams];
  __shared__ int kind[kMaxBeams], bad, n, none;
  __shared__ Partial part[kMaxLists];
  __shared__ Offer list[kMaxTop * kMaxTop], bound, first[kMaxLists], last[kMaxTop];
  const int tid = int(threadIdx.x);
  const int64_t i = blockIdx.x, t0 = i * a.beams;
  const int lists = a.beams * segs, keys = lists * a.top;
  const bool many = lists >= a.top;
  const int deep = many ? 0 : (a.top + lists - 1) / lists - 1;
  const Key* in = seg_top + t0 * segs * a.top;
  // Everything that the first kernel left is asked for before anything is waited for. What
  // beams without tokens left in its place is not looked at.
  Key ahead[kAhead], head[kMaxLists / kJoinThreads], tail = 0;
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if (tid + k * kJoinThreads < keys) ahead[k] = in[tid + k * kJoinThreads];
#pragma unroll
  for (int k = 0; k < kMaxLists / kJoinThreads; ++k) {
    const int l = tid + k * kJoinThreads;
    if (l < lists) {
      head[k] = in[l * a.top + deep];
      part[l] = partial[t0 * segs + l];
    }
  }
  if (!many && tid < lists) tail = in[tid * a.top + a.top - 1];
  float s = -kInf;
  bool done = false;
  if (tid < a.beams) {
    s = a.scores[t0 + tid];
    done = a.finished && a.finished[t0 + tid];
  }
  if (tid == 0) bad = n = none = 0;
  __syncthreads();
  if (tid < a.beams) {
    int k = kNone;
    if (!(s < kInf)) k = kBad;
    else if (s > -kInf && done) k = kFinished;
    else if (s > -kInf) {
      const Partial* p = part + tid * segs;
      float m = p[0].m;
      for (int g = 1; g < segs; ++g) m = fmaxf(m, p[g].m);
      const float scale = scale_of(m);
      double S = 0.0;
      for (int g = 0; g < segs; ++g) S += rescaled(p[g].S, scale_of(p[g].m), scale);
      most[tid] = double(scale);
      log_s[tid] = log(S);
      k = S > 0.0 ? kTokens : S == 0.0 ? kNone : kBad;
    }
    score[tid] = s;
    kind[tid] = k;
    if (k == kBad) bad = 1;
  }
  __syncthreads();
  const int64_t out = i * a.top;
  if (bad) {
    for (int r = tid; r < a.top; r += kJoinThreads) {
      a.score[out + r] = __builtin_nanf("");
      a.parent[out + r] = a.token[out + r] = -1;
    }
    return;
  }
  // Offer `pos` of list l, whose key is `key` if it is one of a token.
  const auto offer = [&](int l, int pos, Key key) {
    const uint32_t b = uint32_t(l / segs);
    Offer o{0, b, 0};
    if (kind[b] == kTokens && key) {
      o.key = key;
      o.total = order_of(double(score[b]) + ((double(key_value(key)) - most[b]) - log_s[b]));
    } else if (kind[b] == kFinished && l % segs == 0 && pos == 0) {
      o.key = 1;
      o.total = order_of(double(score[b]));
    }
    return o;
  };
#pragma unroll
  for (int k = 0; k < kMaxLists / kJoinThreads; ++k) {
    const int l = tid + k * kJoinThreads;
    if (l < lists) {
      first[l] = offer(l, deep, head[k]);
      if (!many && first[l].total == 0) none = 1;   // the worst of them is none
    }
  }
  if (!many && tid < lists) last[tid] = offer(tid, a.top - 1, tail);
  if (tid == 0) bound = Offer{0, 0, 0};
  __syncthreads();
  // A bound that is no offer cuts nothing: every offer stands before it.
  if (many) {
#pragma unroll
    for (int k = 0; k < kMaxLists / kJoinThreads; ++k) {
      const int l = tid + k * kJoinThreads;
      if (l >= lists) continue;
      const Offer mine = first[l];
      int rank = 0;
#pragma unroll 4
      for (int j = 0; j < lists; ++j) rank += first[j].before(mine) ? 1 : 0;
      if (rank == a.top - 1 && mine.total) bound = mine;
    }
  } else if (tid < lists) {
    // the worst of the first ones, if all are offers, and the best of the last ones
    const Offer mine = first[tid], end = last[tid];
    int worse = 0, better = 0;
#pragma unroll 4
    for (int j = 0; j < lists; ++j) {
      worse += mine.before(first[j]) ? 1 : 0;
      better += last[j].before(end) ? 1 : 0;
    }
    if (better == 0 && end.total) bound = end;
    if (worse == 0 && !none) list[0] = mine;
  }
  __syncthreads();
  Offer cut = bound;
  if (!many && !none && list[0].before(cut)) cut = list[0];
  __syncthreads();
#pragma unroll 1
  for (int k = 0; k * kJoinThreads < keys; ++k) {
    const int at = tid + k * kJoinThreads;
    if (at >= keys) break;
    const int l = at / a.top;
    if (many && cut.before(first[l])) continue;   // the whole list lies below
    const Offer o = offer(l, at % a.top, k == 0 ? ahead[0] : k == 1 ? ahead[1] : in[at]);
    if (o.total && !cut.before(o)) list[atomicAdd(&n, 1)] = o;
  }
  __syncthreads();
  const int count = n;
  for (int k = tid; k < count; k += kJoinThreads) {
    const Offer mine = list[k];
    int rank = 0;
#pragma unroll 4
    for (int j = 0; j < count; ++j) rank += list[j].before(mine) ? 1 : 0;
    if (rank >= a.top) continue;
    a.score[out + rank] = float(total_of(mine.total));
    a.parent[out + rank] = mine.beam;
    a.token[out + rank] = kind[mine.beam] == kFinished ? a.pad_token : int64_t(key_index(mine.key));
  }
  for (int r = count + tid; r < a.top; r += kJoinThreads) {
    a.score[out + r] = -kInf;
    a.parent[out + r] = a.token[out + r] = -1;
  }
}

// Segments of a row. The join is there in any case, so rows are cut where they are few, to 2048
// vectors (40 rows of 32000 bf16 16 to 17 us; 1024 20, 4096 16) and 512 workgroups at the most
// (512 rows of 32000 bf16 28 us, up to 256 42; of 131072 37, up to 1024 45).
int segments(int64_t rows, int64_t vocab, int per_vector) {
  const int64_t n = vocab / per_vector;
  return int(std::max<int64_t>(1, std::min<int64_t>({n / 2048, 512 / rows, kMaxSegs})));
}

size_t partial_bytes(int64_t rows, int segs) { return align256(size_t(rows) * segs * sizeof(Partial)); }

constexpr int64_t kMaxBatch = kMaxRows / kMaxBeams;   // sequences of one launch

size_t rows_bytes(int64_t rows, int64_t vocab, int top) {
  const int segs = segments(rows, vocab, 4);   // the type with the most
  return partial_bytes(rows, segs) + align256(size_t(rows) * segs * top * sizeof(Key));
}

// ---------------------------------------------------------------- reordering

// Units of 16 bytes of the pieces' lengths, the last of a piece shorter. A thread takes the
// same unit of all rows of a sequence: it reads those of the parents, then writes, so that a
// tensor can be its own destination, every parent's unit comes from memory once, and rows
// that stay are left alone. Memory bounds it: 32 tensors of four sequences of four beams, 2.65 GB
// read and written, take 540 to 620 us by box and parents (4.1 to 4.9 TB/s), four small ones 7. Of
// one sequence of 16 or 32 beams 3.9 and 4.4 TB/s, of 5 and 8, whose kernel holds 238 registers a
// lane, 2.4 and 2.9; the same in place, less the rows that stay.
struct State {
  const char* src;
  char* dst;
  int64_t src_row, dst_row, src_outer, dst_outer, inner;
  uint32_t per_piece, in_place;
  uint32_t units;         // per_piece x outer
  uint32_t first_block;   // of a sequence's
};
constexpr int kStates = 44;   // below 64
struct States {
  State s[kStates];
  int n;
};
static_assert(sizeof(States) <= 3584, "fits the kernel's arguments");
constexpr int kMoveThreads = 256;

// A number at any byte, and 16 bytes.
template <class T>
struct __attribute__((packed)) Packed {
  T v;
};
typedef uint32x4 uint32x4_byte __attribute__((aligned(1)));

// One unit of every row of a sequence.
template <int NB>
__device__ __forceinline__ void move_unit(const State& s, const char* src, char* dst, uint32_t u,
                                          const int64_t* par, int in_beams, int out_beams) {
  const uint32_t piece = u / s.per_piece;
  const int64_t at = int64_t(u - piece * s.per_piece) * 16;
  src += piece * s.src_outer + at;
  dst += piece * s.dst_outer + at;
  const int64_t left = s.inner - at;
  const auto from = [&](int j) { return par[j] >= 0 && par[j] < in_beams ? par[j] : int64_t(-1); };
  const auto stays = [&](int j) { return s.in_place && par[j] == j; };
  if (left >= 16) {
    uint32x4 v[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      v[j] = uint32x4{0u, 0u, 0u, 0u};
      if (j < out_beams && from(j) >= 0 && !stays(j)) v[j] = *reinterpret_cast<const uint32x4_byte*>(src + from(j) * s.src_row);
    }
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if (j < out_beams && !stays(j)) *reinterpret_cast<uint32x4_byte*>(dst + j * s.dst_row) = v[j];
  } else {   // the piece's end, by the bits of its length
    Packed<uint64_t> v8[NB];
    Packed<uint32_t> v4[NB];
    Packed<uint16_t> v2[NB];
    uint8_t v1[NB];
    const int n = int(left), at4 = n & 8, at2 = n & 12, at1 = n & 14;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      v8[j].v = 0, v4[j].v = 0, v2[j].v = 0, v1[j] = 0;
      if (j < out_beams && from(j) >= 0 && !stays(j)) {
        const char* p = src + from(j) * s.src_row;
        if (n & 8) v8[j] = *reinterpret_cast<const Packed<uint64_t>*>(p);
        if (n & 4) v4[j] = *reinterpret_cast<const Packed<uint32_t>*>(p + at4);
        if (n & 2) v2[j] = *reinterpret_cast<const Packed<uint16_t>*>(p + at2);
        if (n & 1) v1[j] = uint8_t(p[at1]);
      }
    }
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if (j < out_beams && !stays(j)) {
        char* p = dst + j * s.dst_row;
        if (n & 8) *reinterpret_cast<Packed<uint64_t>*>(p) = v8[j];
        if (n & 4) *reinterpret_cast<Packed<uint32_t>*>(p + at4) = v4[j];
        if (n & 2) *reinterpret_cast<Packed<uint16_t>*>(p + at2) = v2[j];
        if (n & 1) p[at1] = char(v1[j]);
      }
  }
}

// A workgroup takes `each` x kMoveThreads neighbouring units of a tensor.
template <int NB>
__global__ void __launch_bounds__(kMoveThreads)
reorder_kernel(States all, int each, const int64_t* __restrict__ parent, int in_beams, int out_beams) {
  const int64_t seq = blockIdx.y;
  int which = 0;   // the last whose first block is not past this one
  for (int step = 32; step > 0; step >>= 1)
    if (which + step < all.n && blockIdx.x >= all.s[which + step].first_block) which += step;
  const State s = all.s[which];
  const char* src = s.src + seq * in_beams * s.src_row;
  char* dst = s.dst + seq * out_beams * s.dst_row;
  const uint32_t u0 = (blockIdx.x - s.first_block) * uint32_t(each * kMoveThreads) + threadIdx.x;
#pragma unroll 1
  for (int k = 0; k < each; ++k) {
    const uint32_t u = u0 + k * kMoveThreads;
    if (u >= s.units) break;
    move_unit<NB>(s, src, dst, u, parent + seq * out_beams, in_beams, out_beams);
  }
}

}  // namespace

size_t beam_select_workspace_bytes(int64_t batch, int beams, int64_t vocab, int top) {
  size_t need = rows_bytes(std::min(batch, kMaxBatch) * beams, vocab, top);
  if (batch > kMaxBatch && batch % kMaxBatch)   // the last launch of many may cut its rows
    need = std::max(need, rows_bytes(batch % kMaxBatch * beams, vocab, top));
  return need;
}

hipError_t launch_beam_select(const BeamArgs& all, int type, void* d_ws, hipStream_t stream) {
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    for (int64_t b = 0; b < all.batch; b += kMaxBatch) {   // the launches share the workspace
      BeamArgs a = all;
      a.batch = std::min(kMaxBatch, all.batch - b);
      a.logits = static_cast<const typename T::raw*>(all.logits) + b * a.beams * a.ld;
      a.scores += b * a.beams;
      if (a.finished) a.finished += b * a.beams;
      a.score += b * a.top, a.parent += b * a.top, a.token += b * a.top;
      const int64_t rows = a.batch * a.beams;
      const int segs = segments(rows, a.vocab, kPerVector<T>);
      Partial* part = static_cast<Partial*>(d_ws);
      Key* keys = reinterpret_cast<Key*>(static_cast<char*>(d_ws) + partial_bytes(rows, segs));
      const uint32_t n = uint32_t(a.vocab) / kPerVector<T>;
      auto go = [&](auto kern, unsigned threads) {
        hipLaunchKernelGGL(kern, dim3(unsigned(rows), unsigned(segs)), dim3(threads), 0, stream, a,
                           uint32_t(segs), (n + segs - 1) / segs, part, keys);
      };
      if (n <= 256) go(beam_rows_kernel<T, 64>, 64);
      else go(beam_rows_kernel<T, 512>, 512);
      hipLaunchKernelGGL(beam_join_kernel, dim3(unsigned(a.batch)), dim3(kJoinThreads), 0, stream, a,
                         segs, part, keys);
    }
    return hipGetLastError();
  });
}

hipError_t launch_beam_reorder(const seedq_beam_state* states, int64_t nstates, const int64_t* d_parent,
                               int64_t batch, int in_beams, int out_beams, hipStream_t stream) {
  constexpr int64_t kMaxBlocks = int64_t(1) << 23;   // of a launch's grid
  // Units of a thread: few where there is little to move, so that every CU has some; the launch
  // is shorter with eight where there is much (8 x 12 beams of 16 tensors 97 us, with one 104).
  double units = 0;
  for (int64_t i = 0; i < nstates; ++i) units += double(states[i].outer) * double(states[i].inner) / 16;
  const int each = int(std::max(1.0, std::min(8.0, units * double(batch) / (kMoveThreads * 2048.0))));
  States all;
  all.n = 0;
  int64_t blocks = 0;
  const auto flush = [&]() {
    for (int64_t b = 0; b < batch && blocks; b += 65535) {
      States part = all;
      for (int i = 0; i < part.n; ++i) {
        part.s[i].src += b * in_beams * part.s[i].src_row;
        part.s[i].dst += b * out_beams * part.s[i].dst_row;
      }
      const dim3 grid(unsigned(blocks), unsigned(std::min<int64_t>(batch - b, 65535)));
      auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, grid, dim3(kMoveThreads), 0, stream, part, each,
                           d_parent + b * out_beams, in_beams, out_beams);
      };
      if (out_beams <= 4) go(reorder_kernel<4>);
      else if (out_beams <= 8) go(reorder_kernel<8>);
      else if (out_beams <= 16) go(reorder_kernel<16>);
      else go(reorder_kernel<32>);
    }
    all.n = 0;
    blocks = 0;
  };
  for (int64_t i = 0; i < nstates; ++i) {
    const seedq_beam_state& s = states[i];
    if (s.outer == 0 || s.inner == 0) continue;
    State d{static_cast<const char*>(s.d_src), static_cast<char*>(s.d_dst), s.src_row, s.dst_row,
            s.src_outer, s.dst_outer, s.inner, 0, s.d_src == s.d_dst ? 1u : 0u, 0, 0};
    int64_t outer = s.outer;
    // Pieces longer than 2^31 bytes, and rows of very many units, are cut.
    for (int64_t o = 0; o < outer;) {
      for (int64_t at = 0; at < s.inner;) {
        const int64_t len = std::min<int64_t>(s.inner - at, int64_t(1) << 31);
        const int64_t per = (len + 15) / 16;
        const int64_t take = len < s.inner ? 1 : std::min<int64_t>(outer - o, std::max<int64_t>(1, (int64_t(1) << 27) / per));
        State e = d;
        e.src += o * s.src_outer + at, e.dst += o * s.dst_outer + at;
        e.inner = len, e.per_piece = uint32_t(per), e.units = uint32_t(per * take);
        const int64_t need = (int64_t(e.units) + each * kMoveThreads - 1) / (each * kMoveThreads);
        if (all.n == kStates || blocks + need > kMaxBlocks) flush();
        e.first_block = uint32_t(blocks);
        all.s[all.n++] = e;
        blocks += need;
        at += len;
        if (at >= s.inner) o += take;
      }
    }
  }
  flush();
  return hipGetLastError();
}

}  // namespace seedq
