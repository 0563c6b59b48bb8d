// Products of a 4-bit matrix with vectors, straight from the codes.
//
// With u the code and z the zero point (8 without), a row's product with x is
//     sum over groups g of s_g sum (u - z_g) x = s_g (sum u x - z_g sum x).
// A byte 0 .. 15 read as an 8-bit float with three mantissa bits stands for u 2^-9 (its
// subnormals and its first binade), so three operations spread the codes of a word over
// bytes and four conversions, which also scale, make eight exact 16-bit floats. Their
// pairs are columns (0, 2), (4, 6), (1, 3), (5, 7); x is put in that order. In fp16 one
// packed addition takes z off exactly. In bf16, which has none, the kernels form sum u x
// and take z sum x from it in fp32 once a group. x in fp32 goes to the matrix core as
// three bf16 pieces of 8 bits (truncated, so that they add up to it exactly) that are
// multiplied like three vectors: every product is exact and only the fp32 sums round.
#include <algorithm>

#include "seedq_ops_device.h"

namespace seedq {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr float kCodeScale = 512.f;   // 2^9

// The 16-bit arithmetic of a kernel. kCentred: codes have their zero point taken off.
struct Half {
  static constexpr bool kCentred = true;
  static constexpr uint32_t kOnes = 0x3C003C00u;
  template <bool HIGH>
  __device__ static __forceinline__ f16x2 pair(uint32_t bytes) {
    return __builtin_bit_cast(
        f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(bytes, kCodeScale, HIGH));
  }
  __device__ static __forceinline__ floatx4 mfma(uint32x4 a, uint32x4 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  __device__ static __forceinline__ floatx16 mfma(uint32x4 a, uint32x4 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
struct Brain {
  static constexpr bool kCentred = false;
  static constexpr uint32_t kOnes = 0x3F803F80u;
  template <bool HIGH>
  __device__ static __forceinline__ bf16x2 pair(uint32_t bytes) {
    return __builtin_bit_cast(
        bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(bytes, kCodeScale, HIGH));
  }
  __device__ static __forceinline__ floatx4 mfma(uint32x4 a, uint32x4 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  __device__ static __forceinline__ floatx16 mfma(uint32x4 a, uint32x4 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};

// The eight codes of a word as 16-bit floats in code order.
template <class M>
__device__ __forceinline__ uint32x4 decode(uint32_t w) {
  const uint32_t even = w & 0x0F0F0F0Fu, odd = (w >> 4) & 0x0F0F0F0Fu;
  return uint32x4{__builtin_bit_cast(uint32_t, M::template pair<false>(even)),
                  __builtin_bit_cast(uint32_t, M::template pair<true>(even)),
                  __builtin_bit_cast(uint32_t, M::template pair<false>(odd)),
                  __builtin_bit_cast(uint32_t, M::template pair<true>(odd))};
}
__device__ __forceinline__ uint32x4 centred(uint32x4 u, f16x2 z) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t pair = u[j];   // a bit cast of a vector's element takes element 0
    u[j] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, pair) - z);
  }
  return u;
}

// Column of element i of the code order.
constexpr int kOrder[8] = {0, 2, 4, 6, 1, 3, 5, 7};
// Eight consecutive 16-bit elements into code order.
__device__ __forceinline__ uint32x4 to_code_order(uint32x4 d) {
  return uint32x4{__builtin_amdgcn_perm(d[1], d[0], 0x05040100u),
                  __builtin_amdgcn_perm(d[3], d[2], 0x05040100u),
                  __builtin_amdgcn_perm(d[1], d[0], 0x07060302u),
                  __builtin_amdgcn_perm(d[3], d[2], 0x07060302u)};
}

// Eight fp32 values as three bf16 pieces in code order.
__device__ __forceinline__ void split8(const float (&f)[8], uint32x4 (&piece)[3]) {
  uint32_t h[3][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float r = f[i];
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      h[p][i] = __builtin_bit_cast(uint32_t, r);
      r -= __builtin_bit_cast(float, h[p][i] & 0xFFFF0000u);
    }
  }
#pragma unroll
  for (int p = 0; p < 3; ++p)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      piece[p][j] = __builtin_amdgcn_perm(h[p][kOrder[2 * j + 1]], h[p][kOrder[2 * j]], 0x07060302u);
}

__device__ __forceinline__ void store_y(void* y, int ytype, int64_t at, float v) {
  if (ytype == SEEDQ_F32) static_cast<float*>(y)[at] = v;
  else static_cast<uint16_t*>(y)[at] = ytype == SEEDQ_F16 ? F16::narrow(v) : BF16::narrow(v);
}

// ---------------------------------------------------------------- few vectors

// One or two vectors, on the vector ALU. A wave holds a slab of columns of x in
// registers, WORDS words of codes a lane, and goes over kRows rows whose codes it reads
// at once; a lane's columns lie in one group, so the scale enters once a lane and row.
// The products u - z (fp16) times x (widened to fp32) are fused multiply-adds that read
// either half of a register. Order of the sums: the columns of a lane, the slabs of a
// wave, the lanes as a tree, the waves one after the other.
constexpr int kRows = 8;
constexpr int kMaxWaves = 16;

template <class X, int NV, int WORDS>
__global__ void __launch_bounds__(64 * kMaxWaves)
gemv_few_kernel(Q4 q, const typename X::raw* __restrict__ x, int64_t ldx, int slabs,
                void* __restrict__ y, int ytype, int64_t ldy) {
  __shared__ float part[kMaxWaves][NV][kRows];
  const int lane = int(threadIdx.x & 63), wave = int(threadIdx.x >> 6), waves = int(blockDim.x >> 6);
  const int64_t r0 = int64_t(blockIdx.x) * kRows;
  float acc[NV][kRows] = {};
  for (int slab = wave; slab < slabs; slab += waves) {
    const int64_t w0 = (int64_t(slab) * 64 + lane) * WORDS;
    const int64_t wl = w0 * kC < q.ncols ? w0 : 0;   // idle lanes: the row's start, x as zeros
    const int64_t g = wl * kC >> q.gshift;
    uint32_t code[kRows][WORDS];
    float s[kRows], z[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int64_t r = std::min(r0 + i, q.nrows - 1);
      const uint32_t* p = q.codes + r * q.row_words + wl;
      if constexpr (WORDS == 4) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        code[i][0] = v.x, code[i][1] = v.y, code[i][2] = v.z, code[i][3] = v.w;
      } else if constexpr (WORDS == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        code[i][0] = v.x, code[i][1] = v.y;
      } else {
        code[i][0] = *p;
      }
      s[i] = F16::widen(q.scale[r * q.ngroups + g]);
      z[i] = q.zero ? float(q.zero[r * q.ngroups + g] & 15) : 8.f;
    }
    float xf[NV][WORDS][8];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int w = 0; w < WORDS; ++w) {
        const int64_t c = (w0 + w) * kC;
        const typename X::raw* xv = x + v * ldx + c;
#pragma unroll
        for (int i = 0; i < 8; ++i) xf[v][w][i] = 0.f;
        if (c < q.ncols) load8<X>(xv, xf[v][w]);
      }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      float d[NV] = {};
      const f16x2 zz = {_Float16(z[i]), _Float16(z[i])};
#pragma unroll
      for (int w = 0; w < WORDS; ++w) {
        const uint32x4 u = centred(decode<Half>(code[i][w]), zz);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t bits = u[j];
          const f16x2 pair = __builtin_bit_cast(f16x2, bits);
#pragma unroll
          for (int v = 0; v < NV; ++v) {
            d[v] = fmaf(float(pair[0]), xf[v][w][kOrder[2 * j]], d[v]);
            d[v] = fmaf(float(pair[1]), xf[v][w][kOrder[2 * j + 1]], d[v]);
          }
        }
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) acc[v][i] = fmaf(s[i], d[v], acc[v][i]);
    }
  }
  // the eight rows' sums over the lanes: halves of the rows change sides with halves of
  // the lanes, so that lane l ends with row l / 8
#pragma unroll
  for (int v = 0; v < NV; ++v) {
#pragma unroll
    for (int n = kRows / 2, d = 32; n >= 1; n >>= 1, d >>= 1) {
      const bool up = (lane & d) != 0;
#pragma unroll
      for (int k = 0; k < n; ++k) {
        const float keep = up ? acc[v][k + n] : acc[v][k], give = up ? acc[v][k] : acc[v][k + n];
        acc[v][k] = keep + __shfl_xor(give, d, 64);
      }
    }
    float t = acc[v][0];
#pragma unroll
    for (int d = 4; d >= 1; d >>= 1) t += __shfl_xor(t, d, 64);
    if ((lane & 7) == 0) part[wave][v][lane >> 3] = t;
  }
  __syncthreads();
  for (int k = int(threadIdx.x); k < NV * kRows; k += int(blockDim.x)) {
    const int v = k / kRows, i = k % kRows;
    float t = part[0][v][i];
    for (int w = 1; w < waves; ++w) t += part[w][v][i];
    if (r0 + i < q.nrows) store_y(y, ytype, v * ldy + r0 + i, t);
  }
}

// ---------------------------------------------------------------- a batch of vectors

// x in fp32 as three bf16 rows a vector (row 3 v + p), in code order, zeros from ncols
// to the padded end of the codes' rows.
__global__ void __launch_bounds__(256)
split_kernel(const float* __restrict__ x, int64_t ldx, int64_t ncols, int64_t row_words,
             uint16_t* __restrict__ out) {
  const int64_t v = blockIdx.y;
  const int64_t w = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (w >= row_words) return;
  float f[8] = {};
  if (w * kC < ncols) load8<F32>(x + v * ldx + w * kC, f);
  uint32x4 piece[3];
  split8(f, piece);
#pragma unroll
  for (int p = 0; p < 3; ++p)
    *reinterpret_cast<uint32x4*>(out + ((3 * v + p) * row_words + w) * kC) = piece[p];
}

// Up to 16 rows of x (vectors, or a third of a vector in fp32) on the matrix core,
// D = X W^T: a 16x16x32 product takes 16 rows of x and 16 rows of codes. A lane
// reads 16 bytes of codes of row l % 16, columns 32 (l / 16) .. of a chunk of 128. Where
// a group is 128 columns or more, product t takes everybody's word t; in smaller groups
// (NG = 4 or 2 a chunk) the words first change lanes so that product t holds columns
// 32 t .. 32 t + 31 (four lane swaps). Each group's product and, in bf16, sum of x (a
// product with ones) meet in fp32 with the scale and zero point of the lane's row. The waves of
// a workgroup take its chunks in turn and add their sums through LDS in order.
template <int NG, int RT>
struct Chunk {
  uint32x4 code[RT];
  float s[RT][NG], z[RT][NG];
  uint32x4 x[4];
};

template <class M, int P, int NG, int RT>
__global__ void __launch_bounds__(64 * kMaxWaves)
gemv_batch_kernel(Q4 q, int nvec, const uint16_t* __restrict__ x, int64_t ldx,
                  void* __restrict__ y, int ytype, int64_t ldy) {
  extern __shared__ float part[];
  const int lane = int(threadIdx.x & 63), wave = int(threadIdx.x >> 6), waves = int(blockDim.x >> 6);
  const int n = lane & 15, kg = lane >> 4;
  const int64_t r0 = int64_t(blockIdx.x) * (16 * RT);
  const int64_t xcols = P == 3 ? q.row_words * kC : q.ncols;
  const int64_t chunks = (q.ncols + 127) / 128;
  // rows past the last are read as the last and not stored
  const uint16_t* xrow = x + std::min(n, nvec * P - 1) * ldx;
  const uint32_t* crow[RT];
  int64_t grow[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int64_t r = std::min(r0 + 16 * t + n, q.nrows - 1);
    crow[t] = q.codes + r * q.row_words;
    grow[t] = r * q.ngroups;
  }
  auto load = [&](Chunk<NG, RT>& c, int64_t ch) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int64_t w = ch * 16 + kg * 4;
      c.code[t] = uint32x4{0u, 0u, 0u, 0u};
      if (w < q.row_words) c.code[t] = *reinterpret_cast<const uint32x4*>(crow[t] + w);
#pragma unroll
      for (int j = 0; j < NG; ++j) {
        const int64_t g = grow[t] + std::min((ch * 128 + j * (128 / NG)) >> q.gshift, q.ngroups - 1);
        c.s[t][j] = F16::widen(q.scale[g]);
        c.z[t][j] = q.zero ? float(q.zero[g] & 15) : 8.f;
      }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int64_t k = ch * 128 + (NG == 1 ? kg * 32 + t * 8 : t * 32 + kg * 8);
      c.x[t] = uint32x4{0u, 0u, 0u, 0u};
      if (k < xcols) c.x[t] = load16(xrow + k);
    }
  };
  floatx4 sum[RT] = {};
  Chunk<NG, RT> c;
  if (wave < chunks) load(c, wave);
  for (int64_t ch = wave; ch < chunks; ch += waves) {
    Chunk<NG, RT> next = c;
    if (ch + waves < chunks) load(next, ch + waves);
    if constexpr (P == 1)
#pragma unroll
      for (int t = 0; t < 4; ++t) c.x[t] = to_code_order(c.x[t]);
    const uint32x4 ones = {M::kOnes, M::kOnes, M::kOnes, M::kOnes};
    floatx4 xs[NG] = {};
    if constexpr (!M::kCentred)
#pragma unroll
      for (int t = 0; t < 4; ++t) xs[t * NG / 4] = M::mfma(c.x[t], ones, xs[t * NG / 4]);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      uint32x4 w = c.code[t];
      if constexpr (NG > 1) {
        const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
        const auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
        const auto e = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
        const auto f = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
        w = uint32x4{e[0], e[1], f[0], f[1]};
      }
#pragma unroll
      for (int j = 0; j < NG; ++j) {
        floatx4 acc = {};
#pragma unroll
        for (int k = j * 4 / NG; k < (j + 1) * 4 / NG; ++k) {
          uint32x4 u = decode<M>(w[k]);
          if constexpr (M::kCentred) u = centred(u, f16x2{_Float16(c.z[t][j]), _Float16(c.z[t][j])});
          acc = M::mfma(c.x[k], u, acc);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          sum[t][i] = fmaf(c.s[t][j], M::kCentred ? acc[i] : fmaf(-c.z[t][j], xs[j][i], acc[i]),
                           sum[t][i]);
      }
    }
    c = next;
  }
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) part[((wave * RT + t) * 4 + i) * 64 + lane] = sum[t][i];
  __syncthreads();
  // row 4 kg + i of x and row n of the codes lie in lane 16 kg + n, register i
  for (int k = int(threadIdx.x); k < nvec * RT * 16; k += int(blockDim.x)) {
    const int rn = k % (16 * RT), v = k / (16 * RT);
    const int64_t r = r0 + rn;
    float total = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int row = P * v + p;
      const int at = ((rn >> 4) * 4 + (row & 3)) * 64 + (row >> 2) * 16 + (rn & 15);
      float one = part[at];
      for (int w = 1; w < waves; ++w) one += part[w * (RT * 256) + at];
      total += one;
    }
    if (r < q.nrows) store_y(y, ytype, int64_t(v) * ldy + r, total);
  }
}

// ---------------------------------------------------------------- many vectors

// A workgroup of four waves makes 32 MT vectors x 256 rows, a wave 64 of the rows, in
// stages of 128 columns on 32x32x16 products. Every wave decodes its own rows' codes in
// registers (nobody else's), while the vectors' fragments are the same for all four: they
// are laid out once, by frag_kernel, in the order in which lanes take them, so a stage is
// a contiguous piece that goes to LDS without passing registers and is read back without
// bank conflicts. The next stage's fragments and codes are on their way during the
// products. A lane's codes are 16 bytes of row l % 32: columns 32 (l / 32) .. of a chunk of
// 64; product t takes everybody's word t, or, where a group is 32 columns, words that
// have changed lanes so that each half of the chunk has two products of its own.
// Each group's product meets its scale, zero point and sum of x in fp32.
constexpr int kStage = 128;            // columns
constexpr int kTileRows = 256;         // of codes, a workgroup
constexpr int kFragBytes = 1024;       // 64 lanes x 16
constexpr int kStageFrags = 8;         // a stage of 32 vectors, each piece of x
constexpr int kTileVecs = 32;

// What the vectors are made into: fragments [vector tile][stage][piece][8][lane] of 16
// bytes and, for codes that keep their zero point, sums of x [stage][NG][padded vectors].
struct Frags {
  uint32x4* frag;
  float* sums;
  int64_t stages, padded;   // padded: vectors, a multiple of 64
};

// A workgroup: 32 vectors, one stage.
template <class X, int P, bool SUMS, int NG>
__global__ void __launch_bounds__(256)
frag_kernel(const typename X::raw* __restrict__ x, int64_t ldx, int64_t nvec, int64_t ncols, Frags f) {
  __shared__ float part[kTileVecs][17];
  const int64_t stage = blockIdx.x, tile = blockIdx.y;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int item = int(threadIdx.x) + 256 * h;   // 16 neighbours: the 128 columns of a vector
    const int m = item >> 4, w = item & 15;
    const int64_t v = tile * kTileVecs + m, c = stage * kStage + w * kC;
    const bool some = v < nvec && c < ncols;
    uint32x4 piece[3] = {};
    float sum = 0.f;
    if (some) {
      if constexpr (P == 3 || SUMS) {
        float e[8];
        load8<X>(x + v * ldx + c, e);
        sum = ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
        if constexpr (P == 3) split8(e, piece);
      }
      if constexpr (P == 1) piece[0] = to_code_order(load16(x + v * ldx + c));
    }
    const int chunk = w >> 3, k = w & 7;
    const int t = NG == 4 ? k >> 1 : k & 3, lane = (NG == 4 ? k & 1 : k >> 2) * 32 + m;
#pragma unroll
    for (int p = 0; p < P; ++p)
      f.frag[(((tile * f.stages + stage) * P + p) * kStageFrags + chunk * 4 + t) * 64 + lane] = piece[p];
    if (SUMS) part[m][w] = sum;
  }
  if (!SUMS) return;
  __syncthreads();
  if (threadIdx.x < kTileVecs * NG) {
    const int m = int(threadIdx.x) % kTileVecs, j = int(threadIdx.x) / kTileVecs;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16 / NG; ++i) sum += part[m][j * (16 / NG) + i];
    f.sums[(stage * NG + j) * f.padded + tile * kTileVecs + m] = sum;
  }
}

// 16 or 4 bytes a lane to LDS, lane after lane.
__device__ __forceinline__ void to_lds16(const void* from, void* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from),
                                   (__attribute__((address_space(3))) void*)(to), 16, 0, 0);
}
__device__ __forceinline__ void to_lds4(const void* from, void* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from),
                                   (__attribute__((address_space(3))) void*)(to), 4, 0, 0);
}

template <class M, int P, int NG, int MT>
__global__ void __launch_bounds__(256, P == 1 || MT == 1 ? 2 : 1)
gemm_kernel(Q4 q, int64_t nvec, Frags f, int vec_tiles, int row_tiles, int splits,
            void* __restrict__ y, int ytype, int64_t ldy, float* __restrict__ partial) {
  constexpr int kFrags = MT * P * kStageFrags;
  __shared__ __attribute__((aligned(16))) uint32x4 frag[2][kFrags * 64];
  __shared__ __attribute__((aligned(16))) float sums[2][NG][MT * kTileVecs];
  // Workgroups go to the eight XCDs in turn: those of one XCD that run together share
  // their rows' codes in its L2.
  const unsigned id = blockIdx.x, xcd = id & 7, j8 = id >> 3;
  const int vt = int(j8 % unsigned(vec_tiles));
  const int unit = int(j8 / unsigned(vec_tiles)) * 8 + int(xcd);
  if (unit >= row_tiles * splits) return;
  const int rt = unit % row_tiles, split = unit / row_tiles;
  const int s0 = int(f.stages * split / splits), s1 = int(f.stages * (split + 1) / splits);
  const int lane = int(threadIdx.x & 63);
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6));
  const int n = lane & 31, kg = lane >> 5;
  const int64_t r0 = int64_t(rt) * kTileRows + wave * 64;
  const uint32_t* crow[2];
  int64_t grow[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int64_t r = std::min(r0 + 32 * t + n, q.nrows - 1);
    crow[t] = q.codes + r * q.row_words;
    grow[t] = r * q.ngroups;
  }
  struct Rows {
    uint32x4 code[2][2];   // rows' tile, chunk
    float s[2][NG], z[2][NG];
  };
  auto fetch = [&](int stage, int buf, Rows& c) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < kFrags / 4; ++k) {
      const int i = 4 * k + wave;
      const int m = i / (P * kStageFrags), rest = i % (P * kStageFrags);
      const uint32x4* from =
          f.frag + (((vt * MT + m) * f.stages + stage) * int64_t(P * kStageFrags) + rest) * 64 + lane;
      to_lds16(from, &frag[buf][i * 64]);
    }
    if constexpr (!M::kCentred) {
      if (wave < NG && lane < MT * kTileVecs)
        to_lds4(f.sums + (int64_t(stage) * NG + wave) * f.padded + vt * (MT * kTileVecs) + lane,
                &sums[buf][wave][0]);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t w = int64_t(stage) * 16 + h * 8 + kg * 4;
        c.code[t][h] = uint32x4{0u, 0u, 0u, 0u};
        if (w < q.row_words) c.code[t][h] = *reinterpret_cast<const uint32x4*>(crow[t] + w);
      }
#pragma unroll
      for (int j = 0; j < NG; ++j) {
        const int64_t g = grow[t] + std::min((int64_t(stage) * kStage + j * (kStage / NG)) >> q.gshift,
                                             q.ngroups - 1);
        c.s[t][j] = F16::widen(q.scale[g]);
        c.z[t][j] = q.zero ? float(q.zero[g] & 15) : 8.f;
      }
    }
  };
  floatx16 total[2][MT] = {};
  Rows cur;
  fetch(s0, 0, cur);
  for (int s = s0; s < s1; ++s) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this stage's fragments are in LDS
    __syncthreads();                                   // for everybody; the other buffer is free
    const int buf = (s - s0) & 1;
    Rows next = cur;
    if (s + 1 < s1) fetch(s + 1, buf ^ 1, next);
    floatx16 acc[2][MT];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32x4 w[2] = {cur.code[0][h], cur.code[1][h]};
      if constexpr (NG == 4) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const auto a = __builtin_amdgcn_permlane32_swap(w[t][0], w[t][1], false, false);
          const auto b = __builtin_amdgcn_permlane32_swap(w[t][2], w[t][3], false, false);
          w[t] = uint32x4{a[0], b[0], a[1], b[1]};
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        constexpr int kEach = 8 / NG;                // products of a group
        const int at = h * 4 + k, j = at / kEach;
        uint32x4 u[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          u[t] = decode<M>(w[t][k]);
          if constexpr (M::kCentred)
            u[t] = centred(u[t], f16x2{_Float16(cur.z[t][j]), _Float16(cur.z[t][j])});
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int p = 0; p < P; ++p) {
            const uint32x4 a = frag[buf][((m * P + p) * kStageFrags + at) * 64 + lane];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              if (at % kEach == 0 && p == 0) acc[t][m] = M::mfma(a, u[t], floatx16{});
              else acc[t][m] = M::mfma(a, u[t], acc[t][m]);
            }
          }
        if (at % kEach == kEach - 1) {
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
              floatx4 xs = {0.f, 0.f, 0.f, 0.f};
              if constexpr (!M::kCentred)
                xs = *reinterpret_cast<const floatx4*>(&sums[buf][j][m * 32 + 2 * i + 4 * kg]);
#pragma unroll
              for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const float d = M::kCentred ? acc[t][m][i + e]
                                              : fmaf(-cur.z[t][j], xs[e], acc[t][m][i + e]);
                  total[t][m][i + e] = fmaf(cur.s[t][j], d, total[t][m][i + e]);
                }
            }
        }
      }
    }
    cur = next;
  }
  // register i of lane l: vector 8 (i / 4) + 4 (l / 32) + i % 4, row l % 32
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int64_t r = r0 + 32 * t + n;
    if (r >= q.nrows) continue;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int64_t v = int64_t(vt * MT + m) * kTileVecs + 8 * (i >> 2) + 4 * kg + (i & 3);
        if (v >= nvec) continue;
        if (splits > 1) partial[(split * nvec + v) * q.nrows + r] = total[t][m][i];
        else store_y(y, ytype, v * ldy + r, total[t][m][i]);
      }
  }
}

// The splits of the columns added in order.
__global__ void __launch_bounds__(256)
join_kernel(const float* __restrict__ partial, int splits, int64_t nvec, int64_t nrows,
            void* __restrict__ y, int ytype, int64_t ldy) {
  const int64_t v = blockIdx.y;
  const int64_t r = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (r >= nrows) return;
  float sum = 0.f;
  for (int s = 0; s < splits; ++s) sum += partial[(s * nvec + v) * nrows + r];
  store_y(y, ytype, v * ldy + r, sum);
}

// How a product with many vectors is cut.
struct GemmPlan {
  int mt, vec_tiles, row_tiles, splits;
  int64_t stages, padded;
  size_t frag_bytes, sum_bytes, total;
};
GemmPlan gemm_plan(int64_t nrows, int64_t ncols, int64_t nvec, int pieces) {
  GemmPlan p;
  p.mt = nvec <= 32 ? 1 : 2;
  p.vec_tiles = int((nvec + 32 * p.mt - 1) / (32 * p.mt));
  p.row_tiles = int((nrows + kTileRows - 1) / kTileRows);
  p.stages = (ncols + kStage - 1) / kStage;
  p.padded = int64_t(p.vec_tiles) * 32 * p.mt;
  const int64_t tiles = int64_t(p.vec_tiles) * p.row_tiles;
  p.splits = int(std::max<int64_t>(1, std::min<int64_t>(512 / tiles, p.stages / 4)));
  p.frag_bytes = align256(size_t(p.padded / kTileVecs) * p.stages * pieces * kStageFrags * kFragBytes);
  p.sum_bytes = align256(size_t(p.stages) * 4 * p.padded * sizeof(float));
  p.total = p.frag_bytes + p.sum_bytes;
  if (p.splits > 1) p.total += align256(size_t(p.splits) * nvec * nrows * sizeof(float));
  return p;
}

// Vectors of one pass: the grids of the kernels below stay small, and so does the workspace.
constexpr int64_t kMaxVecs = 32768;

template <class X, class M, int P>
hipError_t launch_gemm(const Q4& q, int64_t nvec, const void* d_x, int64_t ldx, void* d_y, int ytype,
                       int64_t ldy, void* d_ws, hipStream_t stream) {
  for (int64_t v = 0; v < nvec; v += kMaxVecs) {
    const int64_t nv = std::min(kMaxVecs, nvec - v);
    const GemmPlan p = gemm_plan(q.nrows, q.ncols, nv, P);
    char* ws = static_cast<char*>(d_ws);
    const Frags f{reinterpret_cast<uint32x4*>(ws), reinterpret_cast<float*>(ws + p.frag_bytes),
                  p.stages, p.padded};
    float* partial = reinterpret_cast<float*>(ws + p.frag_bytes + p.sum_bytes);
    const typename X::raw* x = static_cast<const typename X::raw*>(d_x) + v * ldx;
    void* y = static_cast<char*>(d_y) + v * ldy * (ytype == SEEDQ_F32 ? 4 : 2);
    const unsigned units = unsigned((p.row_tiles * p.splits + 7) / 8 * 8);
    auto go = [&](auto ng, auto mt) {
      constexpr int NG = decltype(ng)::value, MT = decltype(mt)::value;
      hipLaunchKernelGGL((frag_kernel<X, P, !M::kCentred, NG>),
                         dim3(unsigned(p.stages), unsigned(p.padded / kTileVecs)), dim3(256), 0,
                         stream, x, ldx, nv, q.ncols, f);
      hipLaunchKernelGGL((gemm_kernel<M, P, NG, MT>), dim3(units * unsigned(p.vec_tiles)), dim3(256),
                         0, stream, q, nv, f, p.vec_tiles, p.row_tiles, p.splits, y, ytype, ldy,
                         partial);
    };
    auto with_mt = [&](auto ng) {
      p.mt == 1 ? go(ng, std::integral_constant<int, 1>{}) : go(ng, std::integral_constant<int, 2>{});
    };
    if (q.gshift >= 7) with_mt(std::integral_constant<int, 1>{});
    else if (q.gshift == 6) with_mt(std::integral_constant<int, 2>{});
    else with_mt(std::integral_constant<int, 4>{});
    if (p.splits > 1)
      hipLaunchKernelGGL(join_kernel, dim3(unsigned((q.nrows + 255) / 256), unsigned(nv)), dim3(256),
                         0, stream, partial, p.splits, nv, q.nrows, y, ytype, ldy);
  }
  return hipGetLastError();
}

// The ways: up to 2 vectors, up to 16 rows of x on 16x16x32 products, more.
bool few(int64_t nvec) { return nvec <= 2; }
bool batch(int64_t nvec, int xtype) { return nvec * (xtype == SEEDQ_F32 ? 3 : 1) <= 16; }

template <class X>
hipError_t launch_few(const Q4& q, int64_t nvec, const void* d_x, int64_t ldx, void* d_y, int ytype,
                      int64_t ldy, hipStream_t stream) {
  using raw = typename X::raw;
  const int64_t words = (q.ncols + kC - 1) / kC;
  const unsigned grid = unsigned((q.nrows + kRows - 1) / kRows);
  const int per = words > 128 ? 4 : words > 64 ? 2 : 1;
  const int slabs = int((words + 64 * per - 1) / (64 * per));
  const int waves = std::min(slabs, kMaxWaves);
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3(grid), dim3(64 * waves), 0, stream, q, static_cast<const raw*>(d_x),
                       ldx, slabs, d_y, ytype, ldy);
    return hipGetLastError();
  };
  auto words_of = [&](auto nv) {
    constexpr int NV = decltype(nv)::value;
    return per == 4   ? go(gemv_few_kernel<X, NV, 4>)
           : per == 2 ? go(gemv_few_kernel<X, NV, 2>)
                      : go(gemv_few_kernel<X, NV, 1>);
  };
  return nvec == 1 ? words_of(std::integral_constant<int, 1>{})
                   : words_of(std::integral_constant<int, 2>{});
}

template <class M, int P>
hipError_t launch_batch(const Q4& q, int64_t nvec, const uint16_t* x, int64_t ldx, void* d_y, int ytype,
                        int64_t ldy, hipStream_t stream) {
  const int waves = int(std::min<int64_t>(kMaxWaves, (q.ncols + 127) / 128));
  auto go = [&](auto ng, auto rt) {
    constexpr int NG = decltype(ng)::value, RT = decltype(rt)::value;
    hipLaunchKernelGGL((gemv_batch_kernel<M, P, NG, RT>),
                       dim3(unsigned((q.nrows + 16 * RT - 1) / (16 * RT))), dim3(64 * waves),
                       size_t(waves) * RT * 1024, stream, q, int(nvec), x, ldx, d_y, ytype, ldy);
    return hipGetLastError();
  };
  auto with_rt = [&](auto ng) {
    return q.nrows >= 32 * 256 ? go(ng, std::integral_constant<int, 2>{})
                               : go(ng, std::integral_constant<int, 1>{});
  };
  return q.gshift >= 7   ? with_rt(std::integral_constant<int, 1>{})
         : q.gshift == 6 ? with_rt(std::integral_constant<int, 2>{})
                         : with_rt(std::integral_constant<int, 4>{});
}

}  // namespace

// Bytes for up to kMaxRows rows.
static size_t rows_bytes(int64_t nrows, int64_t ncols, int64_t nvec, int xtype) {
  const int pieces = xtype == SEEDQ_F32 ? 3 : 1;
  if (few(nvec)) return 0;
  if (batch(nvec, xtype))
    return pieces == 1 ? 0 : align256(size_t(nvec) * 3 * q4_row_words(ncols) * kC * sizeof(uint16_t));
  // the last pass may be shorter and cut its columns more often
  size_t need = gemm_plan(nrows, ncols, std::min(nvec, kMaxVecs), pieces).total;
  if (nvec > kMaxVecs && nvec % kMaxVecs)
    need = std::max(need, gemm_plan(nrows, ncols, nvec % kMaxVecs, pieces).total);
  return need;
}

size_t q4_gemv_workspace_bytes(int64_t nrows, int64_t ncols, int64_t nvec, int xtype) {
  size_t need = rows_bytes(std::min(nrows, kMaxRows), ncols, nvec, xtype);
  if (nrows > kMaxRows && nrows % kMaxRows)
    need = std::max(need, rows_bytes(nrows % kMaxRows, ncols, nvec, xtype));
  return need;
}

static hipError_t launch_rows(const Q4& q, int64_t nvec, const void* d_x, int xtype, int64_t ldx,
                              void* d_y, int ytype, int64_t ldy, void* d_ws, hipStream_t stream) {
  if (few(nvec))
    return with_type(xtype, [&](auto t) {
      return launch_few<decltype(t)>(q, nvec, d_x, ldx, d_y, ytype, ldy, stream);
    });
  if (!batch(nvec, xtype))
    return xtype == SEEDQ_F32
               ? launch_gemm<F32, Brain, 3>(q, nvec, d_x, ldx, d_y, ytype, ldy, d_ws, stream)
           : xtype == SEEDQ_F16
               ? launch_gemm<F16, Half, 1>(q, nvec, d_x, ldx, d_y, ytype, ldy, d_ws, stream)
               : launch_gemm<BF16, Brain, 1>(q, nvec, d_x, ldx, d_y, ytype, ldy, d_ws, stream);
  if (xtype == SEEDQ_F32) {
    uint16_t* pieces = static_cast<uint16_t*>(d_ws);
    hipLaunchKernelGGL(split_kernel, dim3(unsigned((q.row_words + 255) / 256), unsigned(nvec)),
                       dim3(256), 0, stream, static_cast<const float*>(d_x), ldx, q.ncols,
                       q.row_words, pieces);
    return launch_batch<Brain, 3>(q, nvec, pieces, q.row_words * kC, d_y, ytype, ldy, stream);
  }
  const uint16_t* x = static_cast<const uint16_t*>(d_x);
  return xtype == SEEDQ_F16 ? launch_batch<Half, 1>(q, nvec, x, ldx, d_y, ytype, ldy, stream)
                            : launch_batch<Brain, 1>(q, nvec, x, ldx, d_y, ytype, ldy, stream);
}

hipError_t launch_q4_gemv(const Q4& q, int64_t nvec, const void* d_x, int xtype, int64_t ldx,
                          void* d_y, int ytype, int64_t ldy, void* d_ws, hipStream_t stream) {
  for (int64_t r = 0; r < q.nrows; r += kMaxRows) {
    const hipError_t e =
        launch_rows(q.rows(r), nvec, d_x, xtype, ldx,
                    static_cast<char*>(d_y) + r * (ytype == SEEDQ_F32 ? 4 : 2), ytype, ldy, d_ws, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace seedq
