// Products of a 4-bit matrix with vectors, straight from the codes.
//
// With u the code and z the zero point (8 without), a row's product with x is
//     sum over groups g of s_g sum (u - z_g) x = s_g (sum u x - z_g sum x).
// A byte 0 .. 15 read as an 8-bit float with three mantissa bits stands for u 2^-9 (its
// subnormals and its first binade), so three operations spread the codes of a word over
// bytes and four conversions, which also scale, make eight exact 16-bit floats. They are
// made u 2^-11: a sum over the at most 128 columns that meet before the scale stays within
// 15 / 16 of the largest |x| and cannot overflow where the weights' own products would not;
// what is stored takes the factor back. Their
// pairs are columns (0, 2), (4, 6), (1, 3), (5, 7); x is put in that order. In fp16 one
// packed addition takes z off exactly. In bf16, which has none, the kernels form sum u x
// and take z sum x from it in fp32 once a group; vectors of one sign, whose sums of u x are
// many times the result, cost that form a few units of fp32 (4096 x 4096 and 64 vectors:
// 5e-7 of the result's norm, of both signs 8e-8; sums of the decoded weights' products in
// fp32 4e-7). x in fp32 goes to the matrix core as three bf16 pieces of 8 bits (truncated,
// so that they add up to it exactly) that are multiplied like three vectors, by codes whose
// zero point is taken off byte by byte before the conversion: every product is exact and
// only the fp32 sums round.
#include <algorithm>
#include <type_traits>

#include "seedq_ops_device.h"

namespace seedq {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr float kUnit = 0x1p-11f;             // a code 1 in the products
constexpr float kCodeScale = 512.f * kUnit;
// A zero point as the codes stand in fp16.
__device__ __forceinline__ f16x2 half_zero(float z) {
  const _Float16 h = _Float16(z * kUnit);
  return f16x2{h, h};
}

// The 16-bit arithmetic of a kernel. kCentred: codes have their zero point taken off.
struct Half {
  static constexpr bool kCentred = true;
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
  static constexpr uint32_t kOnes = 0x3A003A00u;   // two of kUnit
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

// bf16 with the zero point off the bytes: 12 operations a word more.
struct Exact : Brain {
  static constexpr bool kCentred = true;
};

// Four bytes as 16-bit floats each, from even and odd codes: a word in code order.
template <class M>
__device__ __forceinline__ uint32x4 to_floats(uint32_t even, uint32_t odd) {
  return uint32x4{__builtin_bit_cast(uint32_t, M::template pair<false>(even)),
                  __builtin_bit_cast(uint32_t, M::template pair<true>(even)),
                  __builtin_bit_cast(uint32_t, M::template pair<false>(odd)),
                  __builtin_bit_cast(uint32_t, M::template pair<true>(odd))};
}
// u - z of four bytes, each as sign and magnitude (an 8-bit float's bits). z: four times.
__device__ __forceinline__ uint32_t differences(uint32_t u, uint32_t z) {
  const uint32_t d = ((u | 0x80808080u) - z) ^ 0x80808080u;   // bytes in two's complement
  const uint32_t minus = d & 0x80808080u, one = minus >> 7;
  return (d ^ (minus - one)) + one;
}
// The eight codes of a word as 16-bit floats in code order, without their zero point where
// M is centred.
template <class M>
__device__ __forceinline__ uint32x4 decode(uint32_t w, float z) {
  const uint32_t even = w & 0x0F0F0F0Fu, odd = (w >> 4) & 0x0F0F0F0Fu;
  if constexpr (std::is_same_v<M, Exact>) {
    const uint32_t zs = uint32_t(z) * 0x01010101u;
    return to_floats<M>(differences(even, zs), differences(odd, zs));
  }
  uint32x4 u = to_floats<M>(even, odd);
  if constexpr (std::is_same_v<M, Half>) {
    const f16x2 zz = half_zero(z);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t pair = u[j];   // a bit cast of a vector's element takes element 0
      u[j] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, pair) - zz);
    }
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

// v: a row's sum, in units of kUnit.
__device__ __forceinline__ void store_y(void* y, int ytype, int64_t at, float v) {
  v *= 1.f / kUnit;
  if (ytype == SEEDQ_F32) static_cast<float*>(y)[at] = v;
  else static_cast<uint16_t*>(y)[at] = ytype == SEEDQ_F16 ? F16::narrow(v) : BF16::narrow(v);
}

// ---------------------------------------------------------------- few vectors

// One or two vectors, or up to four in fp32, on the vector ALU. The vectors lie in LDS (a
// panel of kPanelBytes, which is all of them but for very long rows) and the waves go over the rows: RB
// rows a wave at a time, 2048 columns of them a step, 16 bytes of codes a lane, the next
// steps' codes on their way. A lane's columns lie in one group, so the scale enters once a
// lane and step. The products u - z (fp16) times x are fused multiply-adds in fp32 that read
// either half of a register. Where rows are few, `slices` waves share them, each with
// steps of its own. Order of the sums: the columns of a lane and step, the steps, the
// lanes as a tree, the slices in order.
// Memory bounds one vector (8192 x 28672 fp16 27 to 31 us, 4.0 to 4.4 TB/s of codes and
// scales), the vector ALU more: two take 34 to 38 us, four in fp32 57 to 59, of which half
// an operation a product. 4096 x 4096 takes 5.0 to 5.7 us, 1.9 of them an empty launch.
constexpr int kMaxWaves = 16;
constexpr int kStepCols = 64 * 4 * kC;
constexpr int kPanelBytes = 128 << 10;

template <class X>
struct FewX {   // 8 columns of x as they lie in LDS
  static constexpr int kPlanes = sizeof(typename X::raw) == 4 ? 2 : 1;
  uint32x4 v[kPlanes];
};

template <class X, int NV, int RB, bool ZEROS>
__global__ void __launch_bounds__(64 * kMaxWaves)
gemv_few_kernel(Q4 q, const typename X::raw* __restrict__ x, int64_t ldx, int panel_steps, int slices,
                void* __restrict__ y, int ytype, int64_t ldy) {
  constexpr int kPlanes = FewX<X>::kPlanes;
  extern __shared__ uint32x4 panel[];   // [step][plane][vector][4][64]
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
    int64_t grow[RB];
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      const int64_t r = std::min(r0 + i, q.nrows - 1);
      crow[i] = q.codes + r * q.row_words;
      grow[i] = r * q.ngroups;
    }
    struct Codes {
      uint32x4 code[RB];
      uint16_t s[RB];
      uint8_t z[RB];
    };
    auto fetch = [&](Codes& c, int step) __attribute__((always_inline)) {
      const int64_t w = int64_t(step) * 256 + lane * 4;
      const int64_t wl = w * kC < q.ncols ? w : 0;   // idle lanes: the row's start, x is zero there
      const int64_t g = wl * kC >> q.gshift;
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        c.code[i] = *reinterpret_cast<const uint32x4*>(crow[i] + wl);
        c.s[i] = q.scale[grow[i] + g];
        if (ZEROS) c.z[i] = q.zero[grow[i] + g];   // as it lies in memory: nothing waits for it here
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
          const int at = (w >> 8) * kPlanes * NV * 256 + v * 256 + (w & 3) * 64 + ((w & 255) >> 2);
#pragma unroll
          for (int k = 0; k < kPlanes; ++k) {
            uint32x4 d = {0u, 0u, 0u, 0u};
            if (c < q.ncols) d = load16(x + v * ldx + c + k * 4);
            panel[at + k * NV * 256] = d;
          }
        }
        __syncthreads();
      }
      if (!some) continue;
      auto use = [&](const Codes& c0, int step, Codes& later) __attribute__((always_inline)) {
        fetch(later, std::min(step + 2, to - 1));   // always, so that the wait for c0 is not for it
        float d[NV][RB] = {};
        float z[RB];
#pragma unroll
        for (int i = 0; i < RB; ++i) z[i] = ZEROS ? float(c0.z[i] & 15) : 8.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          float f[NV][8];
#pragma unroll
          for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int k = 0; k < kPlanes; ++k)
              widen<X>(panel[(((step - p0) * kPlanes + k) * NV + v) * 256 + w * 64 + lane], f[v] + 4 * k);
#pragma unroll
          for (int i = 0; i < RB; ++i) {
            const uint32x4 u = decode<Half>(c0.code[i][w], z[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t bits = u[j];
              const f16x2 pair = __builtin_bit_cast(f16x2, bits);
#pragma unroll
              for (int v = 0; v < NV; ++v) {
                d[v][i] = fmaf(float(pair[0]), f[v][kOrder[2 * j]], d[v][i]);
                d[v][i] = fmaf(float(pair[1]), f[v][kOrder[2 * j + 1]], d[v][i]);
              }
            }
          }
        }
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int i = 0; i < RB; ++i) acc[v][i] = fmaf(F16::widen(c0.s[i]), d[v][i], acc[v][i]);
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
        for (int s = 1; s < slices; ++s) total += part[sl * slices + s][v][i];
        const int64_t r = (b0 + sl) * RB + i;
        if (r < q.nrows) store_y(y, ytype, v * ldy + r, total);
      }
      __syncthreads();
    }
  }
}

// ---------------------------------------------------------------- a batch of vectors

// N neighbouring elements of T at any element.
template <class T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
  T at[N];
};

// Up to 16 vectors of 16 bits on the matrix core, D = X W^T: a 16x16x32 product takes 16
// rows of x and 16 rows of codes. A lane reads 16 bytes of codes of row l % 16, columns 32 (l / 16) .. of a chunk of 128. Where
// a group is 128 columns or more, product t takes everybody's word t; in smaller groups
// the words first change lanes so that product t holds columns 32 t .. 32 t + 31 (four
// lane swaps). Each group's product and, in bf16, sum of x (a product with ones) meet in
// fp32 with the scale and zero point of the lane's row. The waves of a workgroup divide
// its columns in blocks of BC chunks and add their sums through LDS in order. A block has
// SB scales a row, which a lane reads at once; its codes are read while the block before
// is multiplied, x a chunk ahead.
// 8192 x 28672 and 8 fp16 vectors take 39 to 45 us (up to 3.1 TB/s of codes). Loads are
// answered in order, so those of x wait behind the next block's codes: where the whole took
// 45 us, it took 36 without them and 26 without decoding as well, which is the memory's. The vectors laid out in LDS instead, for a
// split of the columns each, and the splits joined: 43 to 48 us, at 4096 x 4096 twice as long.
constexpr int kBatchWaves = 8;

template <class M, int BC, int SB, int RT>
__global__ void __launch_bounds__(64 * kBatchWaves)
gemv_batch_kernel(Q4 q, int nvec, const uint16_t* __restrict__ x, int64_t ldx, void* __restrict__ y,
                  int ytype, int64_t ldy) {
  constexpr int NG = SB > BC ? SB / BC : 1;          // groups of a chunk
  constexpr int kSpan = SB < BC ? BC / SB : 1;       // chunks of a group, within the block
  extern __shared__ float part[];
  const int lane = int(threadIdx.x & 63), waves = int(blockDim.x >> 6);
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6));
  const int n = lane & 15, kg = lane >> 4;
  const int64_t r0 = int64_t(blockIdx.x) * (16 * RT);
  const int blocks = int((q.ncols + 128 * BC - 1) / (128 * BC));
  const int b0 = int(int64_t(blocks) * wave / waves), b1 = int(int64_t(blocks) * (wave + 1) / waves);
  // rows past the last are read as the last and not stored
  const uint16_t* xrow = x + std::min(n, nvec - 1) * ldx;
  const uint32_t* crow[RT];
  int64_t grow[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int64_t r = std::min(r0 + 16 * t + n, q.nrows - 1);
    crow[t] = q.codes + r * q.row_words;
    grow[t] = r * q.ngroups;
  }
  struct Block {
    uint32x4 code[RT][BC];
    Pack<uint16_t, SB> s[RT];
    Pack<uint8_t, SB> z[RT];
  };
  auto load = [&](Block& c, int b) __attribute__((always_inline)) {
    const int64_t g0 = int64_t(b) * (BC * 128) >> q.gshift;
    const bool whole = g0 + SB <= q.ngroups;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
      for (int k = 0; k < BC; ++k) {
        const int64_t w = (int64_t(b) * BC + k) * 16 + kg * 4;
        c.code[t][k] = uint32x4{0u, 0u, 0u, 0u};
        if (w < q.row_words) c.code[t][k] = *reinterpret_cast<const uint32x4*>(crow[t] + w);
      }
      const uint16_t* s = q.scale + grow[t];
      const uint8_t* z = q.zero + grow[t];
      if (whole) {
        c.s[t] = *reinterpret_cast<const Pack<uint16_t, SB>*>(s + g0);
        if (q.zero) c.z[t] = *reinterpret_cast<const Pack<uint8_t, SB>*>(z + g0);
      } else {
#pragma unroll
        for (int j = 0; j < SB; ++j) {
          const int64_t g = std::min(g0 + j, q.ngroups - 1);
          c.s[t].at[j] = s[g];
          if (q.zero) c.z[t].at[j] = z[g];
        }
      }
      if (!q.zero)
#pragma unroll
        for (int j = 0; j < SB; ++j) c.z[t].at[j] = 8;
    }
  };
  auto load_x = [&](uint32x4 (&v)[4], int64_t ch) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int64_t k = ch * 128 + (NG == 1 ? kg * 32 + t * 8 : t * 32 + kg * 8);
      v[t] = uint32x4{0u, 0u, 0u, 0u};
      if (k < q.ncols) v[t] = load16(xrow + k);
    }
  };
  floatx4 sum[RT] = {};
  Block c;
  uint32x4 xn[4];
  if (b0 < b1) {
    load(c, b0);
    load_x(xn, int64_t(b0) * BC);
  }
  for (int b = b0; b < b1; ++b) {
    Block next = c;
    if (b + 1 < b1) load(next, b + 1);
#pragma unroll
    for (int ch = 0; ch < BC; ++ch) {
      uint32x4 xc[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) xc[t] = to_code_order(xn[t]);
      load_x(xn, int64_t(b) * BC + ch + 1);
      floatx4 xs[NG] = {};
      if constexpr (!M::kCentred) {
        const uint32x4 ones = {M::kOnes, M::kOnes, M::kOnes, M::kOnes};
#pragma unroll
        for (int t = 0; t < 4; ++t) xs[t * NG / 4] = M::mfma(xc[t], ones, xs[t * NG / 4]);
      }
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        uint32x4 w = c.code[t][ch];
        if constexpr (NG > 1) {
          const auto p0 = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
          const auto p1 = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
          const auto q0 = __builtin_amdgcn_permlane16_swap(p0[0], p1[0], false, false);
          const auto q1 = __builtin_amdgcn_permlane16_swap(p0[1], p1[1], false, false);
          w = uint32x4{q0[0], q0[1], q1[0], q1[1]};
        }
#pragma unroll
        for (int j = 0; j < NG; ++j) {
          const int g = ch * NG / kSpan + j;
          const float s = F16::widen(c.s[t].at[g]), z = float(c.z[t].at[g] & 15);
          floatx4 acc = {};
#pragma unroll
          for (int k = j * 4 / NG; k < (j + 1) * 4 / NG; ++k) {
            acc = M::mfma(xc[k], decode<M>(w[k], z), acc);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
            sum[t][i] = fmaf(s, M::kCentred ? acc[i] : fmaf(-z, xs[j][i], acc[i]), sum[t][i]);
        }
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
    const int at = ((rn >> 4) * 4 + (v & 3)) * 64 + (v >> 2) * 16 + (rn & 15);
    float total = part[at];
    for (int w = 1; w < waves; ++w) total += part[w * (RT * 256) + at];
    if (r < q.nrows) store_y(y, ytype, int64_t(v) * ldy + r, total);
  }
}

// ---------------------------------------------------------------- many vectors

// A workgroup of four waves makes 32 MT vectors x 128 RT rows, a wave 32 RT of the rows, in
// stages of 128 columns on 32x32x16 products. Every wave decodes its own rows' codes in
// registers (nobody else's), while the vectors' fragments are the same for all four: they
// are laid out once, by frag_kernel, in the order in which lanes take them, so a stage is
// a contiguous piece that goes to LDS without passing registers and is read back without
// bank conflicts. The next stage's fragments and codes are on their way during the
// products. A lane's codes are 16 bytes of row l % 32: columns 32 (l / 32) .. of a chunk of
// 64; product t takes everybody's word t, or, where a group is 32 columns, words that
// have changed lanes so that each half of the chunk has two products of its own.
// Each group's product meets its scale, zero point and sum of x in fp32.
// 32000 x 4096 and 512 vectors: 159 to 163 us in fp16, 169 to 184 in bf16 (840 and 790
// TFLOP/s at best), where a library product of the decoded 16-bit matrix takes 100 after 65
// of decoding, and of 2048 vectors 362 after 63 (the codes 660). The scale step is 64
// operations of a wave a group, 128 in bf16, and comes oftener in smaller groups: 64 columns
// take 207 us (229 with zero points), 32 columns 272 (382). In fp32, three products for one,
// 425, in groups of 32 795. What bounds groups of 128 in bf16 is the loads of codes: without
// them the rest took 144 of 172 us, while without decoding or the scales it took 175 and
// without the barriers or the loads to LDS 173. A second stage ahead (three buffers) took
// 190, 16x16x32 products, whose lanes read 64 bytes of a row, 262 (their registers spill).
constexpr int kStage = 128;            // columns
constexpr int kFragBytes = 1024;       // 64 lanes x 16
constexpr int kStageFrags = 8;         // a stage of 32 vectors, each piece of x
constexpr int kTileVecs = 32;

// What the vectors are made into: fragments [vector tile][stage][piece][8][lane] of 16
// bytes and, for codes that keep their zero point, sums of kUnit x [stage][NG][padded vectors].
struct Frags {
  uint32x4* frag;
  float* sums;
  int64_t stages, padded;   // padded: vectors, a multiple of 64
};

// A workgroup: 32 vectors, a stage at a time.
template <class X, int P, bool SUMS, int NG>
__global__ void __launch_bounds__(256)
frag_kernel(const typename X::raw* __restrict__ x, int64_t ldx, int64_t nvec, int64_t ncols, Frags f) {
  __shared__ float part[kTileVecs][17];
  const int64_t tile = blockIdx.y;
  for (int64_t stage = blockIdx.x; stage < f.stages; stage += gridDim.x) {
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
          if constexpr (P == 3) split8(e, piece);
#pragma unroll
          for (int i = 0; i < 8; ++i) e[i] *= kUnit;
          sum = ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
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
    if (!SUMS) continue;
    __syncthreads();
    if (threadIdx.x < kTileVecs * NG) {
      const int m = int(threadIdx.x) % kTileVecs, j = int(threadIdx.x) / kTileVecs;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16 / NG; ++i) sum += part[m][j * (16 / NG) + i];
      f.sums[(stage * NG + j) * f.padded + tile * kTileVecs + m] = sum;
    }
    __syncthreads();   // the next stage's sums go to the same place
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

template <class M, int P, int NG, int MT, int RT>
__global__ void __launch_bounds__(256, P == 1 || MT == 1 ? 2 : 1)
gemm_kernel(Q4 q, int64_t nvec, Frags f, int vec_tiles, int row_tiles, int splits,
            void* __restrict__ y, int ytype, int64_t ldy, float* __restrict__ partial) {
  constexpr int kFrags = MT * P * kStageFrags;
  // Scales and zero points kept as they lie in memory do not wait for their load at once
  // (32000 x 4096 and 512 vectors in groups of 64 256 -> 239 us); in groups of 32 their
  // conversions cost more than that (273 -> 302).
  constexpr bool kRaw = NG < 4;
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
  const int64_t r0 = (int64_t(rt) * 4 + wave) * (32 * RT);
  const uint32_t* crow[RT];
  int64_t grow[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int64_t r = std::min(r0 + 32 * t + n, q.nrows - 1);
    crow[t] = q.codes + r * q.row_words;
    grow[t] = r * q.ngroups;
  }
  struct Rows {
    uint32x4 code[RT][2];   // rows' tile, chunk
    std::conditional_t<kRaw, uint16_t, float> s[RT][NG];
    std::conditional_t<kRaw, uint8_t, float> z[RT][NG];
  };
  auto scale_of = [](auto s) {
    if constexpr (kRaw) return F16::widen(s);
    else return s;
  };
  auto zero_of = [](auto z) {
    if constexpr (kRaw) return float(z & 15);
    else return z;
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
    for (int t = 0; t < RT; ++t) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t w = int64_t(stage) * 16 + h * 8 + kg * 4;
        // past the last column the row's start: x is zero there
        c.code[t][h] = *reinterpret_cast<const uint32x4*>(crow[t] + (w < q.row_words ? w : 0));
      }
#pragma unroll
      for (int j = 0; j < NG; ++j) {
        const int64_t g = grow[t] + std::min((int64_t(stage) * kStage + j * (kStage / NG)) >> q.gshift,
                                             q.ngroups - 1);
        if constexpr (kRaw) {
          c.s[t][j] = q.scale[g];
          c.z[t][j] = q.zero ? q.zero[g] : uint8_t(8);
        } else {
          c.s[t][j] = F16::widen(q.scale[g]);
          c.z[t][j] = q.zero ? float(q.zero[g] & 15) : 8.f;
        }
      }
    }
  };
  floatx16 total[RT][MT] = {};
  Rows cur;
  fetch(s0, 0, cur);
  for (int s = s0; s < s1; ++s) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this stage's fragments are in LDS
    __syncthreads();                                   // for everybody; the other buffer is free
    const int buf = (s - s0) & 1;
    Rows next = cur;
    if (s + 1 < s1) fetch(s + 1, buf ^ 1, next);
    // The pieces after the first have sums of their own: added to its sums, which are 2^8
    // times theirs, each would cost a rounding of the whole.
    floatx16 acc[RT][MT], low[P == 1 ? 1 : RT][P == 1 ? 1 : MT];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32x4 w[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) w[t] = cur.code[t][h];
      if constexpr (NG == 4) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const auto a = __builtin_amdgcn_permlane32_swap(w[t][0], w[t][1], false, false);
          const auto b = __builtin_amdgcn_permlane32_swap(w[t][2], w[t][3], false, false);
          w[t] = uint32x4{a[0], b[0], a[1], b[1]};
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        constexpr int kEach = 8 / NG;                // products of a group
        const int at = h * 4 + k, j = at / kEach;
        uint32x4 u[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) u[t] = decode<M>(w[t][k], zero_of(cur.z[t][j]));
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int p = 0; p < P; ++p) {
            const uint32x4 a = frag[buf][((m * P + p) * kStageFrags + at) * 64 + lane];
#pragma unroll
            for (int t = 0; t < RT; ++t) {
              floatx16& to = p == 0 ? acc[t][m] : low[t][m];
              to = M::mfma(a, u[t], at % kEach == 0 && p < 2 ? floatx16{} : to);
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
              for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  float d = acc[t][m][i + e];
                  if constexpr (P > 1) d += low[t][m][i + e];
                  if constexpr (!M::kCentred) d = fmaf(-zero_of(cur.z[t][j]), xs[e], d);
                  total[t][m][i + e] = fmaf(scale_of(cur.s[t][j]), d, total[t][m][i + e]);
                }
            }
        }
      }
    }
    cur = next;
  }
  // register i of lane l: vector 8 (i / 4) + 4 (l / 32) + i % 4, row l % 32
#pragma unroll
  for (int t = 0; t < RT; ++t) {
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
  int mt, rt, vec_tiles, row_tiles, splits;
  int64_t stages, padded;
  size_t frag_bytes, sum_bytes, total;
};
GemmPlan gemm_plan(int64_t nrows, int64_t ncols, int64_t nvec, int pieces) {
  GemmPlan p;
  p.mt = nvec <= 32 ? 1 : 2;
  p.vec_tiles = int((nvec + 32 * p.mt - 1) / (32 * p.mt));
  // 64 rows a wave need as many tiles as the chip holds workgroups: 32000 x 4096 and 512
  // vectors 169 us (32 rows: 173), in fp32 424 (481); 12000 x 1504 and 300 38.0 (30.1), in
  // fp32 68.5 (58.9), 4096 x 4096 and 64 no difference.
  p.rt = (nrows + 255) / 256 * p.vec_tiles >= 512 ? 2 : 1;
  p.row_tiles = int((nrows + 128 * p.rt - 1) / (128 * p.rt));
  p.stages = (ncols + kStage - 1) / kStage;
  p.padded = int64_t(p.vec_tiles) * 32 * p.mt;
  const int64_t tiles = int64_t(p.vec_tiles) * p.row_tiles;
  // Workgroups for two on each CU, of four stages at least (two in fp32, whose stages take
  // three times the products); each split more is more to join. 8192 x 28672 and 32
  // vectors: up to 512 workgroups 52.2 us, 256 74.4, 1024 56.6; 2000 x 8192 and 17: four
  // stages 16.2, two 20.0; 1001 x 2056 and 100 in fp32: 25.2 and 22.0, but 4096 x 4096 and
  // 64 in fp32 25.2 and 29.2.
  p.splits = int(std::max<int64_t>(
      1, std::min<int64_t>({512 / tiles, p.stages / (pieces == 3 ? 2 : 4), 32})));
  p.frag_bytes = align256(size_t(p.padded / kTileVecs) * p.stages * pieces * kStageFrags * kFragBytes);
  p.sum_bytes = pieces == 3 ? 0 : align256(size_t(p.stages) * 4 * p.padded * sizeof(float));
  p.total = p.frag_bytes + p.sum_bytes;
  if (p.splits > 1) p.total += align256(size_t(p.splits) * nvec * nrows * sizeof(float));
  return p;
}

// Vectors of one pass: the grids of the kernels below stay small, and so does the workspace.
constexpr int64_t kMaxVecs = 32768;
// Stages in one go of frag_kernel: a grid has fewer than 2^32 threads along a dimension, and
// a stage takes 256.
constexpr int64_t kMaxStages = int64_t(1) << 20;

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
    auto go = [&](auto ng, auto mt, auto rt) {
      constexpr int NG = decltype(ng)::value, MT = decltype(mt)::value, RT = decltype(rt)::value;
      hipLaunchKernelGGL((frag_kernel<X, P, !M::kCentred, NG>),
                         dim3(unsigned(std::min(p.stages, kMaxStages)), unsigned(p.padded / kTileVecs)),
                         dim3(256), 0,
                         stream, x, ldx, nv, q.ncols, f);
      hipLaunchKernelGGL((gemm_kernel<M, P, NG, MT, RT>), dim3(units * unsigned(p.vec_tiles)), dim3(256),
                         0, stream, q, nv, f, p.vec_tiles, p.row_tiles, p.splits, y, ytype, ldy,
                         partial);
    };
    auto with_mt = [&](auto ng) {
      using One = std::integral_constant<int, 1>;
      using Two = std::integral_constant<int, 2>;
      if (p.mt == 1) p.rt == 1 ? go(ng, One{}, One{}) : go(ng, One{}, Two{});
      else p.rt == 1 ? go(ng, Two{}, One{}) : go(ng, Two{}, Two{});
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

// The ways: the vector ALU, 16x16x32 products, the tiles for many vectors. In fp32 the
// first takes up to four vectors at a time (14336 x 4096 and 4 19.6 us, the tiles 21.9; at
// worst 8192 x 28672 and 4 56.7 and 53.8), twice where the codes are few (4096 x 4096 and
// 5 13.1 and 16.6, and 8 16.5 and 16.2; 8192 x 4096 and 5 19.4 and 17.4). In 16 bits it
// takes two, which a batch would do in less where the codes are many (8192 x 28672 in bf16
// 38 and 33 us, 14336 x 4096 14.3 and 13.8), and the batch 16 (32000 x 4096 29.2 us, the
// tiles 27.8; 4096 x 4096 8.1 and 13.7).
enum class Way { kFew, kBatch, kMany };
Way way(int64_t nrows, int64_t ncols, int64_t nvec, int xtype) {
  if (xtype == SEEDQ_F32)
    return nvec <= 4 || (nvec <= 8 && nrows * ncols <= int64_t(1) << 24) ? Way::kFew : Way::kMany;
  return nvec <= 2 ? Way::kFew : nvec <= 16 ? Way::kBatch : Way::kMany;
}

template <class X>
hipError_t launch_few(const Q4& q, int64_t nvec, const void* d_x, int64_t ldx, void* d_y, int ytype,
                      int64_t ldy, hipStream_t stream) {
  using raw = typename X::raw;
  const int64_t steps = (q.ncols + kStepCols - 1) / kStepCols;
  auto go = [&](auto kern, int nv, int rb, int64_t v) {
    const size_t step_bytes = size_t(nv) * kStepCols * sizeof(raw);
    const int panel_steps = int(std::min<int64_t>(steps, kPanelBytes / step_bytes));
    const int64_t batches = (q.nrows + rb - 1) / rb;
    // Few rows of many columns are shared by several waves (100 x 28672 5.6 us, one wave a
    // row 9.7).
    const int slices = int(std::max<int64_t>(
        1, std::min<int64_t>({1024 / batches, panel_steps >= 4 ? panel_steps : 1, 8})));
    // Large workgroups where the panel is large, small ones where rows are few: one vector
    // with 16, 8 and 4 waves takes 27.6, 28.8 and 41.4 us at 8192 x 28672 in fp16, 5.4,
    // 5.1 and 5.1 at 4096 x 4096 in bf16, 5.2, 3.9 and 3.5 at 1001 x 2056.
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
    // Two rows a wave share what is read of x: 32000 x 4096 18.9 us (one row 22.4), 8192 x
    // 28672 and two vectors 34.5 (36.7), four in fp32 58.3 (70.6); 14336 x 4096 and one
    // vector 11.6 (11.2), in fp32 10.9 (9.6).
    const bool two = q.nrows >= 16384 || (NV > 1 && q.nrows >= 8192);
    if (q.zero) two ? go(gemv_few_kernel<X, NV, 2, true>, NV, 2, v) : go(gemv_few_kernel<X, NV, 1, true>, NV, 1, v);
    else two ? go(gemv_few_kernel<X, NV, 2, false>, NV, 2, v) : go(gemv_few_kernel<X, NV, 1, false>, NV, 1, v);
  };
  for (int64_t v = 0; v < nvec; v += 4) {
    const int64_t n = nvec - v;
    if (n == 1) rows(std::integral_constant<int, 1>{}, v);
    else if (n == 2) rows(std::integral_constant<int, 2>{}, v);
    else if constexpr (sizeof(raw) == 4)
      n == 3 ? rows(std::integral_constant<int, 3>{}, v) : rows(std::integral_constant<int, 4>{}, v);
  }
  return hipGetLastError();
}

template <class M>
hipError_t launch_batch(const Q4& q, int64_t nvec, const uint16_t* x, int64_t ldx, void* d_y, int ytype,
                        int64_t ldy, hipStream_t stream) {
  // Two tiles of rows a workgroup, which share what is read of x, where that leaves every
  // CU a workgroup: 8192 x 28672 and 8 vectors 44 us (one tile 58), 4096 x 4096 and 4 7.8
  // (5.8). With many workgroups four waves: 32000 x 4096 and 8 24.2 (eight 29.8).
  const bool two = q.nrows >= 32 * 256;
  auto go = [&](auto bc, auto sb) {
    constexpr int BC = decltype(bc)::value, SB = decltype(sb)::value;
    auto launch = [&](auto kern, int rt) {
      const int64_t groups = (q.nrows + 16 * rt - 1) / (16 * rt), blocks = (q.ncols + 128 * BC - 1) / (128 * BC);
      const int waves = int(std::min<int64_t>(blocks, groups >= 512 ? 4 : kBatchWaves));
      hipLaunchKernelGGL(kern, dim3(unsigned(groups)), dim3(64 * waves), size_t(waves) * rt * 1024,
                         stream, q, int(nvec), x, ldx, d_y, ytype, ldy);
    };
    two ? launch(gemv_batch_kernel<M, BC, SB, 2>, 2) : launch(gemv_batch_kernel<M, BC, SB, 1>, 1);
    return hipGetLastError();
  };
  using std::integral_constant;
  const integral_constant<int, 4> four;
  switch (q.gshift) {
    case 5: return go(integral_constant<int, 2>{}, integral_constant<int, 8>{});
    case 6: return go(four, integral_constant<int, 8>{});
    case 7: return go(four, integral_constant<int, 4>{});
    case 8: return go(four, integral_constant<int, 2>{});
    default: return go(four, integral_constant<int, 1>{});
  }
}

}  // namespace

// Bytes for up to kMaxRows rows.
static size_t rows_bytes(int64_t nrows, int64_t ncols, int64_t nvec, int xtype) {
  if (way(nrows, ncols, nvec, xtype) != Way::kMany) return 0;
  const int pieces = xtype == SEEDQ_F32 ? 3 : 1;
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
  switch (way(q.nrows, q.ncols, nvec, xtype)) {
    case Way::kFew:
      return with_type(xtype, [&](auto t) {
        return launch_few<decltype(t)>(q, nvec, d_x, ldx, d_y, ytype, ldy, stream);
      });
    case Way::kBatch: {
      const uint16_t* x = static_cast<const uint16_t*>(d_x);
      return xtype == SEEDQ_F16 ? launch_batch<Half>(q, nvec, x, ldx, d_y, ytype, ldy, stream)
                                : launch_batch<Brain>(q, nvec, x, ldx, d_y, ytype, ldy, stream);
    }
    default:
      return xtype == SEEDQ_F32
                 ? launch_gemm<F32, Exact, 3>(q, nvec, d_x, ldx, d_y, ytype, ldy, d_ws, stream)
             : xtype == SEEDQ_F16
                 ? launch_gemm<F16, Half, 1>(q, nvec, d_x, ldx, d_y, ytype, ldy, d_ws, stream)
                 : launch_gemm<BF16, Brain, 1>(q, nvec, d_x, ldx, d_y, ytype, ldy, d_ws, stream);
  }
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
