// Products of a matrix of microscaled 4-bit floats with vectors of 16 or 32 bits, straight
// from the codes.
//
// A code times its block's power of two has two significant bits and fp32's range, so bf16
// holds it: one conversion instruction makes two exact weights, exponent included, and the
// matrix core adds their products up over blocks without a scale step. Vectors enter as
// bf16 pieces that add up to them exactly: one of bf16, two of fp16 (11 bits), three of
// fp32 (24), multiplied like as many vectors. Every product is exact and only the fp32
// sums round.
#include <algorithm>
#include <type_traits>

#include "seedq_mx4_internal.h"
#include "seedq_mx4_device.h"

namespace seedq {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

// Two of the weights of a word; which is a constant where this is inlined.
__device__ __forceinline__ bf16x2 pair_of(uint32_t w, float scale, int which) {
  return which == 0   ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)
         : which == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)
         : which == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)
                      : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
}

// The eight weights of a word.
__device__ __forceinline__ bf16x8 decode(uint32_t w, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Pieces of a type, and the rows of a product that a vector takes up.
template <class X>
constexpr int kPieces = std::is_same_v<X, BF16> ? 1 : std::is_same_v<X, F16> ? 2 : 3;
template <class X>
constexpr int kSpan = std::is_same_v<X, BF16> ? 1 : std::is_same_v<X, F16> ? 2 : 4;

// Eight consecutive elements as pieces, each the upper 16 bits of what is left: truncated,
// so that the next piece is exact too.
template <class X>
__device__ __forceinline__ void split8(const typename X::raw* p, uint32x4 (&piece)[kPieces<X>]) {
  if constexpr (std::is_same_v<X, BF16>) {
    piece[0] = load16(p);
  } else {
    float f[8];
    load8<X>(p, f);
#pragma unroll
    for (int k = 0; k < kPieces<X>; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t lo = __builtin_bit_cast(uint32_t, f[2 * j]);
        const uint32_t hi = __builtin_bit_cast(uint32_t, f[2 * j + 1]);
        piece[k][j] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
        f[2 * j] -= __builtin_bit_cast(float, lo & 0xFFFF0000u);
        f[2 * j + 1] -= __builtin_bit_cast(float, hi & 0xFFFF0000u);
      }
  }
}

// ---------------------------------------------------------------- few vectors

// On the vector ALU. The vectors lie in LDS (a panel of kFewBytes, which is all of them but
// for very long rows) and the waves go over the rows: RB rows a wave at a time, 2048 columns
// of them a step, a block of 16 bytes of codes and its exponent a lane, the next two steps'
// on their way. In 16 bits two products a dot instruction, whose sum is fp32. Where rows are
// few, `slices` waves share them, each with steps of its own. Order of the sums: the columns
// of a lane, step after step, the lanes as a tree, the slices in order.
// Memory bounds one vector (8192 x 28672 in bf16 24.7 us, 5.1 TB/s of codes and exponents;
// 32000 x 4096 15.1, 4.6 TB/s), the vector ALU more: two vectors take 27.8 us, two of fp32,
// an operation a product, 31.5. 4096 x 4096 takes 4.5, some 2 of them an empty launch. A
// batch's kernel takes 30.5, 16.3 and 5.5 us for one vector: its loads touch 16 rows each.
constexpr int kMaxWaves = 16;
constexpr int kStepCols = 64 * kMxBlock;
constexpr int kFewBytes = 128 << 10;

// acc += the eight products of a word. Weights as fp16 leave the exponent to the caller:
// their range does not hold it.
template <class X>
__device__ __forceinline__ float dot8(uint32_t w, float scale, const uint32x4* x, float acc) {
  if constexpr (std::is_same_v<X, BF16>) {
    const bf16x8 xs = __builtin_bit_cast(bf16x8, x[0]), ws = decode(w, scale);
#pragma unroll
    for (int i = 0; i < 8; i += 2)
      acc = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{ws[i], ws[i + 1]}, bf16x2{xs[i], xs[i + 1]}, acc, false);
  } else if constexpr (std::is_same_v<X, F16>) {
    const f16x8 xs = __builtin_bit_cast(f16x8, x[0]);
    const f16x2 ws[4] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 0),
                         __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 1),
                         __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 2),
                         __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 3)};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      acc = __builtin_amdgcn_fdot2(ws[i], f16x2{xs[2 * i], xs[2 * i + 1]}, acc, false);
  } else {
    const floatx2 ws[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0),
                           __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1),
                           __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2),
                           __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3)};
    const floatx4 lo = __builtin_bit_cast(floatx4, x[0]), hi = __builtin_bit_cast(floatx4, x[1]);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = fmaf(ws[i / 2][i % 2], lo[i], acc);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = fmaf(ws[2 + i / 2][i % 2], hi[i], acc);
  }
  return acc;
}

template <class X, int NV, int RB>
__global__ void __launch_bounds__(64 * kMaxWaves)
few_kernel(Mx4 q, const typename X::raw* __restrict__ x, int64_t ldx, int panel_steps, int slices,
           void* __restrict__ y, int ytype, int64_t ldy) {
  constexpr int kPlanes = sizeof(typename X::raw) == 4 ? 2 : 1;   // 16-byte vectors of 8 columns
  extern __shared__ uint32x4 lds[];   // [step][vector][word][lane][plane]
  __shared__ float part[kMaxWaves][NV][RB];
  const int lane = int(threadIdx.x & 63);
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6));
  const int slots = int(blockDim.x >> 6) / slices, slot = wave / slices, slice = wave % slices;
  const int steps = int((q.ncols + kStepCols - 1) / kStepCols);
  const int64_t batches = (q.nrows + RB - 1) / RB;
  for (int64_t b0 = int64_t(blockIdx.x) * slots; b0 < batches; b0 += int64_t(gridDim.x) * slots) {
    const int64_t r0 = (b0 + slot) * RB;
    const bool some = r0 < q.nrows;
    const uint32_t* crow[RB];
    const uint8_t* srow[RB];
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      const int64_t r = std::min(r0 + i, q.nrows - 1);
      crow[i] = q.codes + r * q.row_words;
      srow[i] = q.scale + r * q.nblocks;
    }
    struct Codes {
      uint32x4 code[RB];
      uint8_t s[RB];
    };
    const auto fetch = [&](Codes& c, int step) __attribute__((always_inline)) {
      // idle lanes: the row's last block again, whose x is zero here
      const int64_t block = std::min(int64_t(step) * 64 + lane, q.nblocks - 1);
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        c.code[i] = *reinterpret_cast<const uint32x4*>(crow[i] + block * 4);
        c.s[i] = srow[i][block];   // as it lies in memory: nothing waits for it here
      }
    };
    float acc[NV][RB] = {};
    for (int p0 = 0; p0 < steps; p0 += panel_steps) {
      const int p1 = std::min(p0 + panel_steps, steps), n = p1 - p0;
      const int from = p0 + n * slice / slices, to = p0 + n * (slice + 1) / slices;
      Codes c0, c1, c2;
      if (some && from < to) {
        fetch(c0, from);
        fetch(c1, std::min(from + 1, to - 1));
      }
      if (steps > panel_steps || b0 == int64_t(blockIdx.x) * slots) {
        __syncthreads();   // the panel before is done with
        for (int i = int(threadIdx.x); i < n * 256 * NV; i += int(blockDim.x)) {
          const int v = i / (n * 256), w = i % (n * 256);   // word w of the panel
          const int64_t c = (int64_t(p0) * 256 + w) * kC;
          const int at = (((w >> 8) * NV + v) * 4 + (w & 3)) * 64 * kPlanes + ((w & 255) >> 2) * kPlanes;
#pragma unroll
          for (int k = 0; k < kPlanes; ++k) {
            uint32x4 d = {0u, 0u, 0u, 0u};
            if (c < q.ncols) d = load16(x + v * ldx + c + k * 4);
            lds[at + k] = d;
          }
        }
        __syncthreads();
      }
      if (!some) continue;
      const auto use = [&](const Codes& c, int step, Codes& later) __attribute__((always_inline)) {
        fetch(later, std::min(step + 2, to - 1));   // always, so that the wait for c is not for it
        float d[NV][RB] = {}, s[RB];
#pragma unroll
        for (int i = 0; i < RB; ++i) s[i] = mx_scale(c.s[i]);
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int v = 0; v < NV; ++v) {
            uint32x4 xs[kPlanes];
#pragma unroll
            for (int k = 0; k < kPlanes; ++k)
              xs[k] = lds[((((step - p0) * NV + v) * 4 + w) * 64 + lane) * kPlanes + k];
#pragma unroll
            for (int i = 0; i < RB; ++i)
              if constexpr (std::is_same_v<X, F16>) d[v][i] = dot8<X>(c.code[i][w], s[i], xs, d[v][i]);
              else acc[v][i] = dot8<X>(c.code[i][w], s[i], xs, acc[v][i]);
          }
        if constexpr (std::is_same_v<X, F16>)
#pragma unroll
          for (int i = 0; i < RB; ++i) {
            // 2^-127 is no number without its mantissa, and the NaN one none without it
            const float f = c.s[i] == 0 ? 0x1p-127f : c.s[i] == 255 ? __builtin_nanf("") : s[i];
#pragma unroll
            for (int v = 0; v < NV; ++v) acc[v][i] = fmaf(f, d[v][i], acc[v][i]);
          }
      };
      for (int step = from; step < to; step += 3) {
        use(c0, step, c2);
        if (step + 1 >= to) break;
        use(c1, step + 1, c0);
        if (step + 2 >= to) break;
        use(c2, step + 2, c1);
      }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        acc[v][i] = lanes_reduce(acc[v][i], [](float a, float b) { return a + b; });
        if (slices > 1) {
          if (lane == 0) part[wave][v][i] = acc[v][i];
        } else if (lane == 0 && r0 + i < q.nrows) {
          store_y(y, ytype, v * ldy + r0 + i, acc[v][i]);
        }
      }
    if (slices > 1) {
      __syncthreads();
      for (int k = int(threadIdx.x); k < slots * NV * RB; k += int(blockDim.x)) {
        const int i = k % RB, sl = k / RB % slots, v = k / RB / slots;
        float total = part[sl * slices][v][i];
        for (int t = 1; t < slices; ++t) total += part[sl * slices + t][v][i];
        const int64_t r = (b0 + sl) * RB + i;
        if (r < q.nrows) store_y(y, ytype, v * ldy + r, total);
      }
      __syncthreads();
    }
  }
}

template <class X>
hipError_t launch_few(const Mx4& q, int64_t nvec, const void* d_x, int64_t ldx, void* d_y, int ytype,
                      int64_t ldy, hipStream_t stream) {
  using raw = typename X::raw;
  const int64_t steps = (q.ncols + kStepCols - 1) / kStepCols;
  auto go = [&](auto kern, int nv, int rb, int64_t v) {
    const size_t step_bytes = size_t(nv) * kStepCols * sizeof(raw);
    const int panel_steps = int(std::min<int64_t>(steps, kFewBytes / step_bytes));
    const int64_t batches = (q.nrows + rb - 1) / rb;
    // Few rows of many columns are shared by several waves: 100 x 28672 4.9 us, one wave a row 7.5.
    const int slices = int(std::max<int64_t>(
        1, std::min<int64_t>({1024 / batches, panel_steps >= 4 ? panel_steps : 1, 8})));
    // Large workgroups where the panel is large, small ones where rows are few: one bf16 vector with
    // 16, 8 and 4 waves takes 25.5, 26.1 and 36.6 us at 8192 x 28672, 4.4, 4.5 and 4.7 at 4096 x
    // 4096, three of fp32 7.2, 5.3 and 5.3 at 1001 x 2056.
    int waves = batches >= 4096 && panel_steps * step_bytes > (32 << 10) ? 16 : batches >= 2048 ? 8 : 4;
    waves = std::max(waves, slices) / slices * slices;
    const int slots = waves / slices;
    const unsigned grid = unsigned(std::min<int64_t>((batches + slots - 1) / slots, 4096 / waves));
    hipLaunchKernelGGL(kern, dim3(grid), dim3(64 * waves), panel_steps * step_bytes, stream, q,
                       static_cast<const raw*>(d_x) + v * ldx, ldx, panel_steps, slices,
                       static_cast<char*>(d_y) + v * ldy * (ytype == SEEDQ_F32 ? 4 : 2), ytype, ldy);
  };
  auto rows = [&](auto nv, int64_t v) {
    constexpr int NV = decltype(nv)::value;
    // Two rows a wave share what is read of x: 32000 x 4096 15.0 us (one row 17.0), and two
    // vectors 18.3 (20.1); 14336 x 4096 and two 10.8 (9.7), 1001 x 2056 and three of fp32 6.2 (5.3).
    // Three and four vectors come with up to 8192 rows only, or with rows so long that there are
    // fewer than 4096.
    if constexpr (NV <= 2)
      if (q.nrows >= 16384) return go(few_kernel<X, NV, 2>, NV, 2, v);
    go(few_kernel<X, NV, 1>, NV, 1, v);
  };
  for (int64_t v = 0; v < nvec; v += 4) {
    const int64_t n = nvec - v;
    if (n == 1) rows(std::integral_constant<int, 1>{}, v);
    else if (n == 2) rows(std::integral_constant<int, 2>{}, v);
    else if (n == 3) rows(std::integral_constant<int, 3>{}, v);
    else rows(std::integral_constant<int, 4>{}, v);
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------- up to a few tiles of vectors

// D = X W^T in 16x16x32 products: 16 rows of pieces, 16 rows of codes. The columns are cut
// into panels (blockIdx.y) of chunks of 128, whose pieces lie in LDS for as long as the
// workgroup goes over rows. A wave takes 16 RT rows and a slice of the panel: a lane reads
// the 16 bytes of block l / 16 of a chunk of row l % 16, which one exponent scales, and
// product t takes everybody's word t; a step of kDeep chunks is on its way while the one
// before is multiplied with the pieces from LDS. Row i of a product lies in lanes 16 (i / 4) .., register i % 4,
// so the pieces of a vector, which are neighbouring rows, meet in a lane. Slices meet in LDS
// in order, panels in the join kernel.
// Memory bounds it: 8192 x 28672 and 8 fp16 vectors take 26 us and the join 5 (4.8 TB/s of
// codes and exponents while it runs), 16 of bf16 34.5 in all, 32 46; 4096 x 4096 and 8 7.5.
// The cut matters as much as the code: with panels of 96 KB and 16 rows a wave throughout,
// which left waves without rows, the first took 48. Exponents read a byte a lane and chunk
// took 10 us more of 41.
constexpr int kChunk = 128;
constexpr int kDeep = 4;   // chunks of a step

struct Cut {
  int chunks, panel_chunks;   // of a row, of a panel
  int slices, groups;         // waves of a workgroup: slices x groups of rows
};

template <class X, int XT, int RT>
__global__ void __launch_bounds__(XT == 1 ? 1024 : 512)
batch_kernel(Mx4 q, int nvec, const typename X::raw* __restrict__ x, int64_t ldx, Cut cut,
             void* __restrict__ y, int ytype, int64_t ldy, float* __restrict__ partial) {
  constexpr int P = kPieces<X>, kEach = 16 / kSpan<X>;   // vectors of a tile
  extern __shared__ uint32x4 lds[];
  const int lane = int(threadIdx.x & 63), n = lane & 15, kg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6));
  const int slice = wave % cut.slices, group = wave / cut.slices;
  const int c0 = int(blockIdx.y) * cut.panel_chunks;
  const int cn = std::min(cut.panel_chunks, cut.chunks - c0);
  const int rows_x = P * nvec;
  int xrow[XT];   // rows past the last vector are read as the last and not stored
#pragma unroll
  for (int t = 0; t < XT; ++t)
    xrow[t] = kg * rows_x + std::min(t * kEach + n / kSpan<X>, nvec - 1) * P +
              std::min(n % kSpan<X>, P - 1);
  const int steps = (cn + kDeep - 1) / kDeep;
  const int from = steps * slice / cut.slices * kDeep, to = std::min(cn, steps * (slice + 1) / cut.slices * kDeep);
  const int64_t tiles = (q.nrows + 16 * RT - 1) / (16 * RT);
  const uint32_t* crow[RT];
  const uint8_t* srow[RT];
  struct Codes {
    uint32x4 code[kDeep][RT], s[RT];
  };
  const auto rows = [&](int64_t r0) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int64_t r = std::min(r0 + 16 * t + n, q.nrows - 1);
      crow[t] = q.codes + r * q.row_words;
      srow[t] = q.scale + r * q.nblocks;
    }
  };
  const auto load = [&](Codes& k, int c) __attribute__((always_inline)) {
    const int64_t b0 = int64_t(c0 + c) * 4;   // q.nblocks >= 16
#pragma unroll
    for (int d = 0; d < kDeep; ++d) {
      // past the last block the last one again, of the same row: its x is zero
      const int64_t block = std::min(b0 + 4 * d + kg, q.nblocks - 1);
#pragma unroll
      for (int t = 0; t < RT; ++t) k.code[d][t] = *reinterpret_cast<const uint32x4*>(crow[t] + block * 4);
    }
    // the exponents of the step's 16 blocks, the same for the four lanes of a row
#pragma unroll
    for (int t = 0; t < RT; ++t) k.s[t] = *reinterpret_cast<const uint32x4_byte*>(srow[t] + std::min(b0, q.nblocks - 16));
  };
  Codes k0, k1;   // the first step's are on their way while x is laid out
  int64_t b = int64_t(blockIdx.x) * cut.groups;
  rows((b + group) * (16 * RT));
  load(k0, from);
  // [chunk][word][block][vector and piece]
  for (int i = int(threadIdx.x); i < cn * 16 * nvec; i += int(blockDim.x)) {
    const int v = i / (cn * 16), k = i % (cn * 16);   // neighbours: columns of a vector
    const int64_t c = (int64_t(c0) * 16 + k) * kC;
    uint32x4 piece[P] = {};
    if (c < q.ncols) split8<X>(x + v * ldx + c, piece);
    const int at = (((k >> 4) * 4 + (k & 3)) * 4 + ((k >> 2) & 3)) * rows_x + v * P;
#pragma unroll
    for (int p = 0; p < P; ++p) lds[at + p] = piece[p];
  }
  __syncthreads();
  for (; b < tiles; b += int64_t(gridDim.x) * cut.groups) {
    const int64_t r0 = (b + group) * (16 * RT);
    const bool some = b + group < tiles;
    floatx4 acc[XT][RT] = {};
    const auto use = [&](const Codes& k, int c) __attribute__((always_inline)) {
      uint32x4 se[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) se[t] = after_bytes(k.s[t], int64_t(c0 + c) * 4 + 16 - q.nblocks);
#pragma unroll
      for (int d = 0; d < kDeep; ++d) {
        if (c + d >= to) break;
        const uint32x4* xs = lds + (c + d) * 16 * rows_x;
        float s[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) s[t] = mx_scale(__builtin_amdgcn_ubfe(se[t][d], 8 * kg, 8));
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          bf16x8 a[XT];
#pragma unroll
          for (int t = 0; t < XT; ++t) a[t] = __builtin_bit_cast(bf16x8, xs[w * 4 * rows_x + xrow[t]]);
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            const bf16x8 u = decode(k.code[d][r][w], s[r]);
#pragma unroll
            for (int t = 0; t < XT; ++t)
              acc[t][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[t], u, acc[t][r], 0, 0, 0);
          }
        }
      }
    };
    for (int c = from; some && c < to; c += 2 * kDeep) {
      if (c + kDeep < to) load(k1, c + kDeep);
      use(k0, c);
      if (c + kDeep >= to) break;
      if (c + 2 * kDeep < to) load(k0, c + 2 * kDeep);
      use(k1, c + kDeep);
    }
    const int64_t next = b + int64_t(gridDim.x) * cut.groups;
    if (next < tiles) {   // the next rows' first step
      rows((next + group) * (16 * RT));
      load(k0, from);
    }
    // vectors of a lane: the sums of their pieces, the smallest first
    constexpr int kMine = 4 / kSpan<X>;
    float sum[XT][RT][kMine];
#pragma unroll
    for (int t = 0; t < XT; ++t)
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
          float v = acc[t][r][i * kSpan<X> + P - 1];
#pragma unroll
          for (int p = P - 2; p >= 0; --p) v += acc[t][r][i * kSpan<X> + p];
          sum[t][r][i] = v;
        }
    if (cut.slices > 1) {
      float* part = reinterpret_cast<float*>(lds + int64_t(cut.panel_chunks) * 16 * rows_x);
      constexpr int kSums = XT * RT * kMine;
#pragma unroll
      for (int t = 0; t < XT; ++t)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int i = 0; i < kMine; ++i)
            part[(wave * kSums + (t * RT + r) * kMine + i) * 64 + lane] = sum[t][r][i];
      __syncthreads();
      if (slice == 0)
        for (int w = 1; w < cut.slices; ++w)
#pragma unroll
          for (int t = 0; t < XT; ++t)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
              for (int i = 0; i < kMine; ++i)
                sum[t][r][i] += part[((wave + w) * kSums + (t * RT + r) * kMine + i) * 64 + lane];
      __syncthreads();
    }
    if (!some || slice != 0) continue;
#pragma unroll
    for (int t = 0; t < XT; ++t)
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
          const int v = t * kEach + kg * kMine + i;
          const int64_t row = r0 + 16 * r + n;
          if (v >= nvec || row >= q.nrows) continue;
          if (gridDim.y > 1) partial[(int64_t(blockIdx.y) * nvec + v) * q.nrows + row] = sum[t][r][i];
          else store_y(y, ytype, v * ldy + row, sum[t][r][i]);
        }
  }
}

// ---------------------------------------------------------------- many vectors

// A workgroup of four waves makes 32 MT vectors x 128 RT rows, a wave 32 RT of the rows, in
// stages of 64 C columns on 32x32x16 products. Every wave decodes its own rows' codes in
// registers, while the vectors' fragments are the same for all four: they are laid out once,
// by frag_kernel, in the order in which lanes take them, so a stage is a contiguous piece
// that goes to LDS without passing registers and is read back without bank conflicts. The
// next stage's fragments and codes are on their way during the products. A lane's codes are
// the 16 bytes of block l / 32 of a chunk of 64 columns of row l % 32; product t takes
// everybody's word t.
// 32000 x 4096 and 512 bf16 vectors take 119 to 128 us (1.05 to 1.13 PFLOP/s by box) after 6
// for the fragments, of fp16 198, of fp32 318; a library product of the decoded 16-bit matrix
// takes 97. Zero data takes 13 % less: the matrix core's power counts. Neither loads (all from
// one stage: no change) nor the barrier bound it (one between two steps, with the next
// stage's first fragments read before the last products: no change), but what is done for
// every 128 vectors again, conversions and loads of codes, and 10 us of results that all
// workgroups write at the end. Fragments read right before their use took 142, the next
// stage's loads issued together 137; 64 vectors a tile take 164, one tile of rows a wave 133.
constexpr int kFrags = 4;       // of 64 lanes x 16 bytes: a chunk of 64 columns, 32 vectors, each piece
constexpr int kTileVecs = 32;

// A workgroup: 32 vectors, four chunks at a time. Fragments
// [vector tile][chunk][piece, the smallest first][4][lane].
template <class X>
__global__ void __launch_bounds__(256)
frag_kernel(const typename X::raw* __restrict__ x, int64_t ldx, int64_t nvec, int64_t ncols,
            int64_t chunks, uint32x4* __restrict__ frag) {
  constexpr int P = kPieces<X>;
  const int64_t tile = blockIdx.y;
  // 32 neighbours: the words of four chunks of a vector
  const int w = int(threadIdx.x & 31), k = w & 7;
  for (int64_t c4 = int64_t(blockIdx.x) * 4; c4 < chunks; c4 += int64_t(gridDim.x) * 4) {
    const int64_t chunk = c4 + (w >> 3), c = chunk * 64 + k * kC;
    if (chunk >= chunks) continue;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const int m = int(threadIdx.x >> 5) + 8 * h;
      const int64_t v = tile * kTileVecs + m;
      uint32x4 piece[P] = {};
      if (v < nvec && c < ncols) split8<X>(x + v * ldx + c, piece);
#pragma unroll
      for (int p = 0; p < P; ++p)
        frag[(((tile * chunks + chunk) * P + (P - 1 - p)) * kFrags + (k & 3)) * 64 + (k >> 2) * 32 + m] = piece[p];
    }
  }
}

template <int P, int MT, int RT, int C>
__global__ void __launch_bounds__(256, 2)
gemm_kernel(Mx4 q, int64_t nvec, const uint32x4* __restrict__ frags, int64_t chunks, int vec_tiles,
            int row_tiles, int splits, void* __restrict__ y, int ytype, int64_t ldy,
            float* __restrict__ partial) {
  constexpr int kEach = P * kFrags;             // fragments of a chunk and tile of vectors
  __shared__ __attribute__((aligned(16))) uint32x4 lds[2][C * MT * kEach * 64];
  // Workgroups go to the eight XCDs in turn: those of one XCD that run together share
  // their rows' codes in its L2.
  const unsigned id = blockIdx.x, xcd = id & 7, j8 = id >> 3;
  const int vt = int(j8 % unsigned(vec_tiles));
  const int unit = int(j8 / unsigned(vec_tiles)) * 8 + int(xcd);
  if (unit >= row_tiles * splits) return;
  const int rt = unit % row_tiles, split = unit / row_tiles;
  const int64_t stages = chunks / C;
  const int64_t s0 = stages * split / splits, s1 = stages * (split + 1) / splits;
  const int lane = int(threadIdx.x & 63);
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6));
  const int n = lane & 31, kg = lane >> 5;
  const int64_t r0 = (int64_t(rt) * 4 + wave) * (32 * RT);
  const uint32_t* crow[RT];
  const uint8_t* srow[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int64_t r = std::min(r0 + 32 * t + n, q.nrows - 1);
    crow[t] = q.codes + r * q.row_words;
    srow[t] = q.scale + r * q.nblocks;
  }
  struct Rows {
    uint32x4 code[RT][C];
    uint8_t s[RT][C];   // as they lie in memory: nothing waits for them at once
  };
  // The loads of a stage one by one: fragments, codes, exponents.
  constexpr int kDma = C * MT * kEach / 4, kLoads = kDma + 2 * RT * C;
  const auto fetch = [&](int64_t stage, int buf, Rows& k, int i) __attribute__((always_inline)) {
    if (i < kDma) {
      const int f = 4 * i + wave;   // [chunk][tile][piece][4]
      const int c = f / (MT * kEach), m = f / kEach % MT, rest = f % kEach;
      const int64_t chunk = stage * C + c;
      to_lds16(frags + ((int64_t(vt * MT + m) * chunks + chunk) * kEach + rest) * 64 + lane, &lds[buf][f * 64]);
      return;
    }
    const int t = (i - kDma) % RT, c = (i - kDma) / RT % C;
    // past the last block the last one again, of the same row: its x is zero
    const int64_t block = std::min((stage * C + c) * 2 + kg, q.nblocks - 1);
    if (i < kDma + RT * C) k.code[t][c] = *reinterpret_cast<const uint32x4*>(crow[t] + block * 4);
    else k.s[t][c] = srow[t][block];
  };
  floatx16 acc[RT][MT] = {};
  Rows cur;
#pragma unroll
  for (int i = 0; i < kLoads; ++i) fetch(s0, 0, cur, i);
  for (int64_t s = s0; s < s1; ++s) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this stage's fragments are in LDS
    __syncthreads();                                   // for everybody; the other buffer is free
    const int buf = int(s - s0) & 1;
    Rows next;
    const int64_t later = std::min(s + 1, s1 - 1);   // always, so that there is no branch
    // Step (c, k) is 16 columns of each half of a chunk. Its fragments and weights are made
    // ready between the products of the step before, in the order in which they are needed:
    // left to itself the compiler reads a fragment right before its use. The next stage's
    // loads are issued one by one between the first products.
    bf16x8 a[2][MT * P];
    bf16x2 w[2][RT][4];
    float scale[RT][C];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int c = 0; c < C; ++c) scale[t][c] = mx_scale(cur.s[t][c]);
    const auto fragment = [&](int i, int m) __attribute__((always_inline)) {
      a[i & 1][m] = __builtin_bit_cast(
          bf16x8, lds[buf][(((i / 4) * MT * P + m) * kFrags + i % 4) * 64 + lane]);
    };
    const auto convert = [&](int i, int j) __attribute__((always_inline)) {
      const int t = j / 4;
      w[i & 1][t][j % 4] = pair_of(cur.code[t][i / 4][i % 4], scale[t][i / 4], j % 4);
    };
#pragma unroll
    for (int m = 0; m < MT * P; ++m) fragment(0, m);
#pragma unroll
    for (int j = 0; j < 4 * RT; ++j) convert(0, j);
#pragma unroll
    for (int i = 0; i < 4 * C; ++i)
#pragma unroll
      for (int m = 0; m < MT * P; ++m) {
        constexpr int kGroups = 4 * C * MT * P;
        for (int l = (i * MT * P + m) * 2 * kLoads / kGroups; l < (i * MT * P + m + 1) * 2 * kLoads / kGroups; ++l)
          if (l < kLoads) fetch(later, buf ^ 1, next, l);
        if (i + 1 < 4 * C) {
          fragment(i + 1, m);
#pragma unroll
          for (int j = 4 * RT * m / (MT * P); j < 4 * RT * (m + 1) / (MT * P); ++j) convert(i + 1, j);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const bf16x2* u = w[i & 1][t];
          acc[t][m / P] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              a[i & 1][m], bf16x8{u[0][0], u[0][1], u[1][0], u[1][1], u[2][0], u[2][1], u[3][0], u[3][1]},
              acc[t][m / P], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    cur = next;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing is on its way to LDS when it is given up
  // register i of lane l: vector 8 (i / 4) + 4 (l / 32) + i % 4, row l % 32
  const auto write = [&](auto type, auto whole, void* to, int64_t ld) __attribute__((always_inline)) {
    using Y = decltype(type);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int64_t r = r0 + 32 * t + n;
      if (r >= q.nrows) continue;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int64_t v0 = int64_t(vt * MT + m) * kTileVecs + 4 * kg;
        typename Y::raw* p = static_cast<typename Y::raw*>(to) + v0 * ld + r;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if (decltype(whole)::value || v0 + 8 * (i >> 2) + (i & 3) < nvec) *p = Y::narrow(acc[t][m][i]);
          p += (i & 3) == 3 ? 5 * ld : ld;
          __builtin_amdgcn_sched_barrier(0);   // one address at a time
        }
      }
    }
  };
  const auto write_as = [&](auto type, void* to, int64_t ld) __attribute__((always_inline)) {
    if (int64_t(vt + 1) * MT * kTileVecs <= nvec) write(type, std::true_type{}, to, ld);
    else write(type, std::false_type{}, to, ld);
  };
  if (splits > 1) write_as(F32{}, partial + split * nvec * q.nrows, q.nrows);
  else if (ytype == SEEDQ_F32) write_as(F32{}, y, ldy);
  else if (ytype == SEEDQ_F16) write_as(F16{}, y, ldy);
  else write_as(BF16{}, y, ldy);
}

constexpr size_t kLdsBytes = 160 << 10;
constexpr int kWorkgroups = 256;
constexpr int kMaxPanels = 32;

struct BatchPlan {
  Cut cut;
  int xt, rt, panels, waves;
  unsigned grid;
  size_t lds, partial;
};
// The cut that the following model finds fastest, in us. A wave goes through its chunks at
// its share of the memory's rate, 1 KB RT in 0.84 RT with all waves at work, but no faster
// than its loads in flight, its CU's part of that rate and the CU's LDS allow, and starts and
// ends the sums of each of its rows; a workgroup lays out its panel; panels cost a second
// launch and its traffic.
BatchPlan batch_plan(int64_t nrows, int64_t ncols, int64_t nvec, int xtype) {
  const int pieces = xtype == SEEDQ_F32 ? 3 : xtype == SEEDQ_F16 ? 2 : 1;
  const int each = xtype == SEEDQ_F32 ? 4 : xtype == SEEDQ_F16 ? 8 : 16;
  BatchPlan best{};
  const int xt = nvec <= each ? 1 : nvec <= 2 * each ? 2 : 4, rt = xt == 2 ? 2 : 1;
  const int most = xt == 1 ? 16 : 8;
  const int64_t chunk_bytes = int64_t(pieces) * nvec * 256;
  const int chunks = int((ncols + kChunk - 1) / kChunk);
  const int64_t tiles = (nrows + 16 * rt - 1) / (16 * rt);
  const size_t part = size_t(xt) * rt * 1024 * each / 16;   // of a wave, where slices meet
  double least = 0.0;
  const auto consider = [&](int panels, int groups) {
    BatchPlan p;
    p.cut.chunks = chunks;
    p.cut.panel_chunks = (chunks + panels - 1) / panels;
    p.panels = (chunks + p.cut.panel_chunks - 1) / p.cut.panel_chunks;
    const int steps = (p.cut.panel_chunks + kDeep - 1) / kDeep;
    const int64_t per_panel = std::max(1, kWorkgroups / p.panels);
    p.cut.groups = groups;
    p.cut.slices = std::max(1, std::min(most / groups, steps));
    p.waves = groups * p.cut.slices;
    p.lds = p.cut.panel_chunks * chunk_bytes + (p.cut.slices > 1 ? p.waves * part : 0);
    if (p.lds > kLdsBytes) return;
    const int64_t units = (tiles + groups - 1) / groups;
    p.grid = unsigned(std::min(units, per_panel));
    const double rounds = double((units + p.grid - 1) / p.grid);
    const double busy = double(p.grid) * p.panels * p.waves / (kWorkgroups * 16.0);
    const double chunk = std::max({0.3, 0.84 * rt * busy, 0.7 * rt * p.waves / 16, 0.015 * xt * p.waves});
    const double us = rounds * (((steps + p.cut.slices - 1) / p.cut.slices) * kDeep * chunk +
                                (p.cut.slices > 1 ? 0.8 : 0.4)) +
                      p.cut.panel_chunks * chunk_bytes / 6e4 +
                      (p.panels > 1 ? 2.5 + p.panels * double(nvec) * nrows * 8 / 5e6 : 0.0);
    if (best.panels && us >= least) return;
    least = us;
    p.xt = xt, p.rt = rt;
    p.partial = p.panels > 1 ? align256(size_t(p.panels) * nvec * nrows * sizeof(float)) : 0;
    best = p;
  };
  const int fit = int(std::max<int64_t>(1, (chunks * chunk_bytes + (128 << 10) - 1) / (128 << 10)));
  for (int panels : {1, 2, 4, 8, 16, 32, fit, fit + 1, fit + 2})
    if (panels >= fit && panels <= std::max(fit, std::min(kMaxPanels, chunks)))
      for (int groups = 1; groups <= most; groups *= 2) consider(panels, groups);
  return best;
}

template <class X>
hipError_t launch_batch(const Mx4& q, int64_t nvec, const void* d_x, int64_t ldx, void* d_y, int ytype,
                        int64_t ldy, void* d_ws, hipStream_t stream) {
  constexpr int xtype = std::is_same_v<X, F32> ? SEEDQ_F32 : std::is_same_v<X, F16> ? SEEDQ_F16 : SEEDQ_BF16;
  const BatchPlan p = batch_plan(q.nrows, q.ncols, nvec, xtype);
  float* partial = static_cast<float*>(d_ws);
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3(p.grid, unsigned(p.panels)), dim3(64 * p.waves), p.lds, stream, q,
                       int(nvec), static_cast<const typename X::raw*>(d_x), ldx, p.cut, d_y, ytype, ldy,
                       partial);
  };
  if (p.xt == 1) go(batch_kernel<X, 1, 1>);
  else if (p.xt == 2) go(batch_kernel<X, 2, 2>);
  else if constexpr (!std::is_same_v<X, BF16>) go(batch_kernel<X, 4, 1>);   // see way
  if (p.panels > 1)
    launch_join(partial, p.panels, nvec, q.nrows, d_y, ytype, ldy, stream);
  return hipGetLastError();
}

// How a product with many vectors is cut.
struct GemmPlan {
  int mt, rt, vec_tiles, row_tiles, splits;
  int64_t chunks;
  size_t frags, total;
};
GemmPlan gemm_plan(int64_t nrows, int64_t ncols, int64_t nvec, int pieces) {
  const int64_t tiles = (nvec + kTileVecs - 1) / kTileVecs;
  GemmPlan best{};
  double least = 0.0;
  // Tiles of vectors of a workgroup: a wider one decodes less often, and the last one may be empty in
  // part; narrow ones fill the chip and are split less. Taken is what the following finds fastest: us
  // of a chunk by x, a workgroup's tiles of pieces, for two workgroups a CU and for one, the join and
  // the fragments. On the mean of 200 sizes it is within 1 % of the fastest width. us by 1, 2, 3 and 4
  //   32000 x 4096, bf16: 5 tiles 107, 74, 59, 66; 8 139, 89, 87, 72; 13 236, 160, 147, 122; 16 272, 175, 156, 128
  //   32000 x 4096, fp16: 5 126, 103, 92, 113; 13 281, 221, 218, 195; fp32 5 147, 140, 131
  //   4096 x 4096, bf16: 4 21.3, 23.8, 23.8, 23.0; 7 30.5, 25.8, 26.1, 26.0; 1001 x 2056 7 14.2, 15.8, 16.5, 17.4
  for (int mt = 1; mt <= (pieces == 3 ? 3 : 4); ++mt) {
    GemmPlan p{};
    p.mt = mt;
    p.vec_tiles = int((tiles + mt - 1) / mt);
    // 64 rows a wave where that leaves as many tiles as the chip holds workgroups: 32000 x 4096 and
    // 512 vectors 123 us (32 rows 133), 14336 x 4096 and 512 84 (66), 4096 x 4096 and 512 43 (35). With
    // nine tiles of pieces the next stage's codes went through scratch memory: 128000 x 4096 and 96
    // fp32 vectors 398 us (32 rows 291).
    const int x = pieces * mt;
    p.rt = (nrows + 255) / 256 * p.vec_tiles >= 400 && x < 9 ? 2 : 1;
    p.row_tiles = int((nrows + 128 * p.rt - 1) / (128 * p.rt));
    p.chunks = (ncols + 127) / 128 * 2;   // whole stages
    const int64_t all = int64_t(p.vec_tiles) * p.row_tiles;
    // Up to two workgroups a CU, of four stages at least: 4096 x 4096 and 300 vectors up to 512
    // workgroups 30.1 us, 256 39.5, 1024 33.2; 4096 x 4096 and 64 four stages 17.5, two 22.4,
    // eight 18.5.
    p.splits = int(std::max<int64_t>(1, std::min<int64_t>({512 / all, p.chunks / 8, 32})));
    p.frags = align256(size_t(p.vec_tiles) * mt * p.chunks * pieces * kFrags * 1024);
    p.total = p.frags;
    if (p.splits > 1) p.total += align256(size_t(p.splits) * nvec * nrows * sizeof(float));
    const double two = p.rt == 1 ? 0.40 + 0.135 * x : 0.72 + 0.265 * x, one = p.rt == 1 ? 0.11 + 0.117 * x : two / 2;
    const int64_t rounds = all * p.splits / 512, rest = all * p.splits % 512;
    const double us = double(p.chunks) / p.splits * (double(rounds) * two + (rest > 256 ? two : rest ? one : 0.0)) +
                      double(p.frags) * 0.85e-6 + (p.splits > 1 ? 5.6 + double(p.total - p.frags) * 0.24e-6 : 0.0);
    if (mt > 1 && us >= least) continue;
    least = us;
    best = p;
  }
  return best;
}

template <class X>
hipError_t launch_gemm(const Mx4& q, int64_t nvec, const void* d_x, int64_t ldx, void* d_y, int ytype,
                       int64_t ldy, void* d_ws, hipStream_t stream) {
  constexpr int P = kPieces<X>, C = P == 1 ? 2 : 1;
  const GemmPlan p = gemm_plan(q.nrows, q.ncols, nvec, P);
  uint32x4* frags = static_cast<uint32x4*>(d_ws);
  float* partial = reinterpret_cast<float*>(static_cast<char*>(d_ws) + p.frags);
  hipLaunchKernelGGL(frag_kernel<X>,
                     dim3(unsigned(std::min<int64_t>((p.chunks + 3) / 4, 65536)), unsigned(p.vec_tiles * p.mt)),
                     dim3(256), 0, stream, static_cast<const typename X::raw*>(d_x), ldx, nvec, q.ncols,
                     p.chunks, frags);
  const int64_t units = (int64_t(p.row_tiles) * p.splits + 7) / 8 * 8;
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3(unsigned(units * p.vec_tiles)), dim3(256), 0, stream, q, nvec, frags,
                       p.chunks, p.vec_tiles, p.row_tiles, p.splits, d_y, ytype, ldy, partial);
  };
  auto with = [&](auto mt) {
    constexpr int MT = decltype(mt)::value;
    if constexpr (P * MT < 9)
      if (p.rt == 2) return go(gemm_kernel<P, MT, 2, C>);
    go(gemm_kernel<P, MT, 1, C>);
  };
  if (p.mt == 1) with(std::integral_constant<int, 1>{});
  else if (p.mt == 2) with(std::integral_constant<int, 2>{});
  else if (p.mt == 3) with(std::integral_constant<int, 3>{});
  else if constexpr (P < 3) with(std::integral_constant<int, 4>{});
  if (p.splits > 1)
    launch_join(partial, p.splits, nvec, q.nrows, d_y, ytype, ldy, stream);
  return hipGetLastError();
}

// The ways, and the vectors of one pass.
constexpr int64_t kMaxVecs = 32768;
// A batch's panels of longer rows than this would be many thousands, and the tiles' fragments
// of few vectors, padded to 32, many times the vectors.
constexpr int64_t kLongRow = int64_t(1) << 22;
enum class Way { kFew, kBatch, kMany };
Way way(int64_t nrows, int64_t ncols, int64_t nvec, int xtype) {
  // The vector ALU takes two vectors, and up to four short ones where rows are few: us by it
  // and by a batch
  //   2 of bf16: 4096 x 4096 5.0 and 6.0, 8192 x 28672 27.8 and 31, 32000 x 4096 18.4 and 16.8
  //   4 of bf16: 4096 x 4096 6.4 and 6.8, 8192 x 28672 35.0 and 31.8, 14336 x 4096 14.9 and 11.4
  //   4 of fp32: 4096 x 4096 8.8 and 7.9, 2000 x 8192 18.4 and 8.4, 8192 x 28672 45.8 and 34.3
  const int size = xtype == SEEDQ_F32 ? 4 : 2;
  if (nvec <= 2 || (nvec <= 4 && nrows <= 8192 && nvec * ncols * size <= 48 << 10)) return Way::kFew;
  // A batch takes two tiles of pieces, and four of fp16 and fp32: us by it and by the tiles for many
  //   32 of bf16: 4096 x 4096 11.4 and 13.6, 8192 x 28672 45.9 and 53.3, 32000 x 4096 30.5 and 35.5
  //   64 of bf16: 4096 x 4096 22.1 and 16.9, 8192 x 28672 109 and 62
  //   32 of fp16: 4096 x 4096 13.4 and 15.8, 8192 x 28672 67.6 and 65.8, 32000 x 4096 40.7 and 45.7
  //   16 of fp32: 4096 x 4096 10.7 and 16.0, 8192 x 28672 51.6 and 72.1, 32000 x 4096 30.7 and 46.1
  const int most = xtype == SEEDQ_F32 ? 16 : 32;
  if (nvec > most || ncols < 16 * kMxBlock) return Way::kMany;   // a batch reads 16 exponents
  return ncols <= kLongRow ? Way::kBatch : Way::kFew;
}
int pieces_of(int xtype) { return xtype == SEEDQ_F32 ? 3 : xtype == SEEDQ_F16 ? 2 : 1; }

// Bytes for up to kMaxRows rows.
size_t rows_bytes(int64_t nrows, int64_t ncols, int64_t nvec, int xtype) {
  switch (way(nrows, ncols, nvec, xtype)) {
    case Way::kFew: return 0;
    case Way::kBatch: return batch_plan(nrows, ncols, nvec, xtype).partial;
    default: break;
  }
  // the last pass may be shorter and cut its columns more often
  size_t need = gemm_plan(nrows, ncols, std::min(nvec, kMaxVecs), pieces_of(xtype)).total;
  if (nvec > kMaxVecs && nvec % kMaxVecs)
    need = std::max(need, gemm_plan(nrows, ncols, nvec % kMaxVecs, pieces_of(xtype)).total);
  return need;
}

}  // namespace

size_t mx4_gemv_workspace_bytes(int64_t nrows, int64_t ncols, int64_t nvec, int xtype) {
  size_t need = rows_bytes(std::min(nrows, kMaxRows), ncols, nvec, xtype);
  if (nrows > kMaxRows && nrows % kMaxRows)
    need = std::max(need, rows_bytes(nrows % kMaxRows, ncols, nvec, xtype));
  return need;
}

hipError_t launch_mx4_gemv(const Mx4& all, int64_t nvec, const void* d_x, int xtype, int64_t ldx,
                           void* d_y, int ytype, int64_t ldy, void* d_ws, hipStream_t stream) {
  const int64_t ysize = ytype == SEEDQ_F32 ? 4 : 2;
  return with_type(xtype, [&](auto t) {
    using X = decltype(t);
    for (int64_t r = 0; r < all.nrows; r += kMaxRows) {
      const Mx4 q = all.rows(r);
      char* y = static_cast<char*>(d_y) + r * ysize;
      hipError_t e = hipSuccess;
      switch (way(q.nrows, q.ncols, nvec, xtype)) {
        case Way::kFew: e = launch_few<X>(q, nvec, d_x, ldx, y, ytype, ldy, stream); break;
        case Way::kBatch: e = launch_batch<X>(q, nvec, d_x, ldx, y, ytype, ldy, d_ws, stream); break;
        default:
          for (int64_t v = 0; v < nvec && e == hipSuccess; v += kMaxVecs)
            e = launch_gemm<X>(q, std::min(kMaxVecs, nvec - v),
                               static_cast<const typename X::raw*>(d_x) + v * ldx, ldx, y + v * ldy * ysize,
                               ytype, ldy, d_ws, stream);
      }
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  });
}

}  // namespace seedq
