// Products of two matrices of microscaled 4-bit floats on the matrix core, which takes the
// codes and the blocks' exponents as they lie in memory: lane l of a 32x32x64 product holds
// the 16 bytes of block l / 32 of row l % 32 and that block's exponent, of a 16x16x128
// product those of block l / 16 of row l % 16.
#include <algorithm>
#include <type_traits>

#include "seedq_mx4_internal.h"
#include "seedq_mx4_device.h"

namespace seedq {
namespace {

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef uint32_t uint32x2 __attribute__((ext_vector_type(2)));

constexpr int kFp4 = 4;   // the instructions' number for the type
__device__ __forceinline__ intx8 fp4_operand(uint32x4 c) {
  return intx8{int(c[0]), int(c[1]), int(c[2]), int(c[3]), 0, 0, 0, 0};
}

// ---------------------------------------------------------------- few rows of A

// 16 AT rows of A against 16 rows of B a workgroup. The waves divide the columns in steps of
// 512, whose codes and exponents a lane reads straight into registers, the next step's
// during the products; their sums meet in LDS in order. A's rows are the same for all
// workgroups and come from the caches. 4 x 4096 x 4096 take 4.3 us, some 2 of them an empty
// launch, 4 x 8192 x 28672 29 (4.3 TB/s), bound by memory; 16 x 8192 x 28672 37, bound by the
// loads of A, where tiles take 33. With 64 rows of A (10.5 us at 4096 x 4096) 16 registers lie in
// scratch memory.
constexpr int kStep = 4;        // products of a step
constexpr int kFewWaves = 8;

template <int AT>
__global__ void __launch_bounds__(64 * kFewWaves)
few_kernel(Mx4 a, Mx4 b, int splits, void* __restrict__ y, int ytype, int64_t ldy, float* __restrict__ partial) {
  __shared__ float part[kFewWaves][AT * 4 * 64];
  const int lane = int(threadIdx.x & 63), n = lane & 15, kg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), waves = int(blockDim.x >> 6);
  const int64_t j0 = int64_t(blockIdx.x) * 16;
  const int64_t steps = (b.nblocks + 4 * kStep - 1) / (4 * kStep);
  const int64_t shares = int64_t(splits) * waves, mine = int64_t(blockIdx.y) * waves + wave;
  const int64_t from = steps * mine / shares, to = steps * (mine + 1) / shares;
  struct Side {
    const uint32_t* codes;
    const uint8_t* scale;
  };
  struct Piece {
    uint32x4 code[kStep], s;
  };
  const int64_t nblocks = b.nblocks;
  const auto row_of = [&](const Mx4& m, int64_t r) __attribute__((always_inline)) {
    r = std::min(r, m.nrows - 1);
    return Side{m.codes + r * m.row_words, m.scale + r * m.nblocks};
  };
  // Past the last block: its codes again under exponent 0 on both sides, which is 2^-254.
  const auto load = [&](const Side& side, Piece& k, int64_t step) __attribute__((always_inline)) {
    const int64_t b0 = step * (4 * kStep);
#pragma unroll
    for (int d = 0; d < kStep; ++d)
      k.code[d] = *reinterpret_cast<const uint32x4*>(side.codes + std::min(b0 + 4 * d + kg, nblocks - 1) * 4);
    k.s = *reinterpret_cast<const uint32x4_byte*>(side.scale + std::min(b0, nblocks - 16));   // nblocks >= 16
  };
  Side arow[AT];
#pragma unroll
  for (int t = 0; t < AT; ++t) arow[t] = row_of(a, 16 * t + n);
  const Side brow = row_of(b, j0 + n);
  floatx4 acc[AT] = {};
  Piece ka[2][AT], kb[2];
  const auto fetch = [&](int buf, int64_t step) __attribute__((always_inline)) {
    load(brow, kb[buf], step);
#pragma unroll
    for (int t = 0; t < AT; ++t) load(arow[t], ka[buf][t], step);
  };
  const auto use = [&](int buf, int64_t step) __attribute__((always_inline)) {
    const int64_t before = (step + 1) * 16 - nblocks;   // in the last step the row's last 16
    kb[buf].s = after_bytes(kb[buf].s, before);
#pragma unroll
    for (int t = 0; t < AT; ++t) ka[buf][t].s = after_bytes(ka[buf][t].s, before);
#pragma unroll
    for (int d = 0; d < kStep; ++d) {
      const int sb = int(kb[buf].s[d] >> (8 * kg));
#pragma unroll
      for (int t = 0; t < AT; ++t)
        acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
            fp4_operand(ka[buf][t].code[d]), fp4_operand(kb[buf].code[d]), acc[t], kFp4, kFp4, 0,
            int(ka[buf][t].s[d] >> (8 * kg)), 0, sb);
    }
  };
  if (from < to) fetch(0, from);
  for (int64_t s = from; s < to; s += 2) {
    if (s + 1 < to) fetch(1, s + 1);
    use(0, s);
    if (s + 1 >= to) break;
    if (s + 2 < to) fetch(0, s + 2);
    use(1, s + 1);
  }
#pragma unroll
  for (int t = 0; t < AT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) part[wave][(t * 4 + i) * 64 + lane] = acc[t][i];
  __syncthreads();
  // row 4 kg + i of A and row n of B lie in lane 16 kg + n, register i
  for (int k = int(threadIdx.x); k < AT * 256; k += int(blockDim.x)) {
    float total = part[0][k];
    for (int w = 1; w < waves; ++w) total += part[w][k];
    const int64_t v = (k >> 8) * 16 + ((k & 63) >> 4) * 4 + ((k >> 6) & 3), r = j0 + (k & 15);
    if (v >= a.nrows || r >= b.nrows) continue;
    if (splits > 1) partial[(int64_t(blockIdx.y) * a.nrows + v) * b.nrows + r] = total;
    else store_y(y, ytype, v * ldy + r, total);
  }
}

// ---------------------------------------------------------------- tiles

// A workgroup of WM x WN waves makes 32 MT WM rows of A x 32 NT WN rows of B, a wave
// 32 MT x 32 NT, in stages of 256 columns: eight blocks, 128 bytes a row, that go to LDS
// without passing registers, the next stage's during the products. Block j of row r lies at
// place j ^ (r / 2 % 8) of the row's eight, so that the 16 bytes that neighbouring lanes
// read, of neighbouring rows, spread over all banks. A lane's four exponents of a stage are
// one register that the products pick their byte of.
// 2048 x 32000 x 4096 take 169 to 188 us by box (2.9 to 3.2 PFLOP/s; the matrix core is busy for 41 %
// of the time), 2048 x 8192 x 28672 250 (3.8), 512 x 14336 x 4096 24, and 29 with codes that come from
// memory. Products alone, without loads, reach 6.7 PFLOP/s on random data
// and 5.2 with as many reads of LDS: power holds them, zeros take a quarter less. What else
// bounds it are the waits at a stage's start. Exponents read by eight bytes of a row a lane took
// 210 us, operands read right before their use 265. Tried and dropped: two workgroups a CU
// with stages of 128 columns (216), the barrier before a stage's last step (registers spill),
// four waves of 128 x 128, one a SIMD (324).
constexpr int kBlocks = 8;   // of a stage

template <int MT, int NT, int WM, int WN, bool SHORT, bool FULL>
__global__ void __launch_bounds__(64 * WM * WN, 2)
tile_kernel(Mx4 a, Mx4 b, int a_tiles, int b_tiles, int splits, void* __restrict__ y, int ytype,
            int64_t ldy, float* __restrict__ partial) {
  constexpr int kWaves = WM * WN, kRowsA = 32 * MT * WM, kRowsB = 32 * NT * WN;
  constexpr int kLoads = (kRowsA + kRowsB) / 8 / kWaves;   // of 8 rows a wave
  static_assert((kRowsA + kRowsB) % (8 * kWaves) == 0 && kRowsA % 8 == 0, "whole loads");
  extern __shared__ uint32x4 lds[];   // [2][kRowsA + kRowsB][8]
  // Workgroups go to the eight XCDs in turn: those of one XCD that run together share
  // rows of B in its L2.
  const unsigned id = blockIdx.x, xcd = id & 7, j8 = id >> 3;
  const int at = int(j8 % unsigned(a_tiles));
  const int unit = int(j8 / unsigned(a_tiles)) * 8 + int(xcd);
  if (unit >= b_tiles * splits) return;
  const int bt = unit % b_tiles, split = unit / b_tiles;
  const int64_t nblocks = b.nblocks, stages = (nblocks + kBlocks - 1) / kBlocks;
  const int64_t s0 = stages * split / splits, s1 = stages * (split + 1) / splits;
  const int lane = int(threadIdx.x & 63), n = lane & 31, kg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6));
  const int wm = wave % WM, wn = wave / WM;
  // FULL: the last tiles are moved up until they are whole (what two make is the same), and
  // so are the stages, so that no row and no block is past the last.
  int64_t i0 = int64_t(at) * kRowsA, j0 = int64_t(bt) * kRowsB;
  if constexpr (FULL) {
    i0 = std::min(i0, a.nrows - kRowsA);
    j0 = std::min(j0, b.nrows - kRowsB);
  }
  // This lane's rows and blocks of the loads: those of a load are a number of rows after the
  // first one's that is the same for all lanes, and the blocks are the same.
  static_assert(kWaves * 8 % 16 == 0, "the swizzle of a load's rows");
  constexpr int kLoadsA = kRowsA / 8 / kWaves;
  const int lrow = wave * 8 + (lane >> 3), lblock = (lane & 7) ^ ((lrow >> 1) & 7);
  const uint32_t* from[FULL ? 1 : kLoads];
  const uint32_t lane_bytes = uint32_t(lrow) * uint32_t(a.row_words * 4) + lblock * 16;   // FULL: fits
  if constexpr (!FULL) {
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int r = k * kWaves * 8 + lrow;
      from[k] = r < kRowsA ? a.codes + std::min(i0 + r, a.nrows - 1) * a.row_words
                           : b.codes + std::min(j0 + r - kRowsA, b.nrows - 1) * b.row_words;
    }
  }
  // Exponents go to LDS sixteen blocks, two stages, at a time, a row a lane: a load of few
  // bytes of many rows costs as much as one of sixteen.
  static_assert(kRowsA + kRowsB == 64 * kWaves, "a row a lane");
  const int srow = wave * 64 + lane;
  const uint8_t* sfrom = srow < kRowsA ? a.scale + std::min(i0 + srow, a.nrows - 1) * nblocks
                                       : b.scale + std::min(j0 + srow - kRowsA, b.nrows - 1) * nblocks;
  uint32x4* const lds_e = lds + 2 * (kRowsA + kRowsB) * 8;   // [2][kRowsA + kRowsB]
  // Past the last block: its codes again under exponent 0 on both sides, which is 2^-254.
  const auto exponents = [&](int64_t stage) __attribute__((always_inline)) {
    const int64_t b0 = stage * kBlocks;
    if constexpr (SHORT) {   // a row is shorter than sixteen bytes
      uint32x4 e = {0u, 0u, 0u, 0u};
      for (int j = 0; j < int(nblocks); ++j) e[j >> 2] |= uint32_t(sfrom[j]) << (8 * (j & 3));
      return e;
    } else {
      return *reinterpret_cast<const uint32x4_byte*>(sfrom + std::min(b0, nblocks - 16));
    }
  };
  const auto of_stage = [&](uint32x4 e, int64_t stage) __attribute__((always_inline)) {
    return after_bytes(e, SHORT ? stage * kBlocks : stage * kBlocks + 16 - nblocks);
  };
  // The loads of a stage one by one.
  const auto fetch = [&](int64_t stage, int buf, int i) __attribute__((always_inline)) {
    const void* at;
    if constexpr (FULL) {   // an address that is the same for all lanes, and the lane's offset
      const uint32_t* all = i < kLoadsA ? a.codes + (i0 + i * kWaves * 8) * a.row_words
                                        : b.codes + (j0 + (i - kLoadsA) * kWaves * 8) * b.row_words;
      at = reinterpret_cast<const char*>(all + stage * (kBlocks * 4)) + lane_bytes;
    } else {
      at = from[i] + std::min(stage * kBlocks + lblock, nblocks - 1) * 4;
    }
    to_lds16(at, &lds[(buf * (kRowsA + kRowsB) + (i * kWaves + wave) * 8) * 8]);
  };
  floatx16 acc[MT][NT] = {};
#pragma unroll
  for (int i = 0; i < kLoads; ++i) fetch(s0, 0, i);
  lds_e[srow] = of_stage(exponents(s0), s0);
  uint32x4 e = {0u, 0u, 0u, 0u};
  const uint32_t pick = kg ? 0x07050301u : 0x06040200u;   // blocks kg, 2 + kg, 4 + kg, 6 + kg
  const int swizzle = (n >> 1) & 7;
  for (int64_t s = s0; s < s1; ++s) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this stage's codes are in LDS
    __syncthreads();                                   // everybody's; the other buffer is free
    const int buf = int(s - s0) & 1;
    const int64_t later = std::min(s + 1, s1 - 1);   // always, so that there is no branch
    const int odd = int(s - s0) & 1, pair = int(s - s0) >> 1 & 1;
    if (!odd && s + 2 < s1) e = exponents(s + 2);
    if (odd) lds_e[(pair ^ 1) * (kRowsA + kRowsB) + srow] = of_stage(e, s + 1);   // read from the next barrier on
    int sc[MT + NT];
    const uint32x2* le = reinterpret_cast<const uint32x2*>(lds_e + pair * (kRowsA + kRowsB)) + odd;
#pragma unroll
    for (int t = 0; t < MT + NT; ++t) {
      const uint32x2 w = le[2 * (t < MT ? (wm * MT + t) * 32 + n : kRowsA + (wn * NT + t - MT) * 32 + n)];
      sc[t] = int(__builtin_amdgcn_perm(w[1], w[0], pick));
    }
    const uint32x4* la = lds + (buf * (kRowsA + kRowsB) + wm * MT * 32 + n) * 8;
    const uint32x4* lb = lds + (buf * (kRowsA + kRowsB) + kRowsA + wn * NT * 32 + n) * 8;
    // The operands of a step of 64 columns are read between the products of the step before,
    // in the order in which they are needed: left to itself the compiler reads them right
    // before their use. The next stage's loads are issued one by one between the first products.
    uint32x4 ca[2][MT], cb[2][NT];
    const auto operand = [&](int k, int o) __attribute__((always_inline)) {
      const int place = (2 * k + kg) ^ swizzle;
      if (o < NT) cb[k & 1][o] = lb[o * 256 + place];
      else ca[k & 1][o - NT] = la[(o - NT) * 256 + place];
    };
    const auto products = [&](auto kk) __attribute__((always_inline)) {
      constexpr int K = decltype(kk)::value;
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          constexpr int kGroups = 4 * MT * NT;   // the loads between the first half of the products
          const int at = K * MT * NT + i * NT + j;
          for (int l = at * 2 * kLoads / kGroups; l < (at + 1) * 2 * kLoads / kGroups; ++l)
            if (l < kLoads) fetch(later, buf ^ 1, l);
          if (K < 3 && i * NT + j < MT + NT) operand(K + 1, i * NT + j);
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
              fp4_operand(ca[K & 1][i]), fp4_operand(cb[K & 1][j]), acc[i][j], kFp4, kFp4, K, sc[i], K, sc[MT + j]);
          __builtin_amdgcn_sched_barrier(0);
        }
    };
    static_assert(MT * NT >= MT + NT, "an operand a product");
#pragma unroll
    for (int o = 0; o < MT + NT; ++o) operand(0, o);
    products(std::integral_constant<int, 0>{});
    products(std::integral_constant<int, 1>{});
    products(std::integral_constant<int, 2>{});
    products(std::integral_constant<int, 3>{});
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing is on its way to LDS when it is given up
  // register e of lane l: row 8 (e / 4) + 4 (l / 32) + e % 4 of A, row l % 32 of B
  const auto write = [&](auto type, void* to, int64_t ld) __attribute__((always_inline)) {
    using Y = decltype(type);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int64_t r = j0 + (wn * NT + j) * 32 + n;
      if (!FULL && r >= b.nrows) continue;
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int64_t v0 = i0 + (wm * MT + i) * 32 + 4 * kg;
        typename Y::raw* p = static_cast<typename Y::raw*>(to) + v0 * ld + r;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int v = 8 * (e >> 2) + (e & 3);
          if (FULL || v0 + v < a.nrows) *p = Y::narrow(acc[i][j][e]);
          p += (e & 3) == 3 ? 5 * ld : ld;
          if (FULL) __builtin_amdgcn_sched_barrier(0);   // one address at a time
        }
      }
    }
  };
  if (splits > 1) write(F32{}, partial + split * a.nrows * b.nrows, b.nrows);
  else if (ytype == SEEDQ_F32) write(F32{}, y, ldy);
  else if (ytype == SEEDQ_F16) write(F16{}, y, ldy);
  else write(BF16{}, y, ldy);
}

// Rows of A of one pass: the grids stay small, and so does the workspace.
constexpr int64_t kMaxVecs = 32768;
constexpr int kFewRows = 64;

struct Plan {
  int tile;   // rows of a tile, 0 for the kernel of few rows
  int a_tiles, b_tiles, splits, waves;
  size_t partial;
};
Plan plan(int64_t na, int64_t nb, int64_t nblocks) {
  Plan p{};
  // The kernel of few rows reads A again for every 16 rows of B and multiplies 16, 32 or 64 of A:
  // us by it and by tiles of 128, the codes of large matrices from memory
  //   4 rows: 131072 x 8192 110 and 135, 32000 x 4096 20.8 and 22.2, 8192 x 28672 28.9 and 32.0
  //   8 rows: 131072 x 8192 123 and 136, 32000 x 4096 22.1 and 22.5, 8192 x 28672 32.1 and 32.1
  //   16 rows: 14336 x 4096 13.4 and 15.7, 1001 x 65536 16.4 and 28.7, 32000 x 4096 23.9 and 23.3, 8192 x
  //     28672 37.2 and 32.8
  //   17 rows: 4096 x 4096 5.3 and 9.6; 32: 4096 x 4096 6.1 and 10.6, 7000 x 4096 10.8 and 11.4, 14336 x
  //     4096 22.7 and 16.9
  //   64 rows: 1001 x 2056 7.0 and 11.1, 4096 x 4096 10.5 and 11.6, 14336 x 4096 38.5 and 19.4
  const double work = double(na <= 16 ? 16 : na <= 32 ? 32 : 64) * double(nb) * double(nblocks * kMxBlock);
  const bool few = na <= 8 || (na <= 16 && work < 1.8e9) || (na <= kFewRows && work < 1.1e9);
  if (few && nblocks >= 16) {
    const int64_t steps = (nblocks + 4 * kStep - 1) / (4 * kStep);
    p.b_tiles = int((nb + 15) / 16);
    p.waves = int(std::min<int64_t>(kFewWaves, steps));
    p.splits = int(std::max<int64_t>(1, std::min<int64_t>({256 / p.b_tiles, steps / (2 * p.waves), 16})));
  } else {
    const int64_t stages = (nblocks + kBlocks - 1) / kBlocks;
    // Times in rounds of 256 tiles of 256, one a CU, of which a last one costs less where it is not
    // whole; 256 tiles of 128, which run two a CU, cost 0.3 of that. us by tiles of 256 and of 128
    //   2048 x 32000 x 4096: 171 and 200, 1024 x 32000 x 4096 80 and 94, 640 x 32000 x 4096 69 and 61
    //   4096 x 4096 x 4096: 43 and 52, 4352 x 4096 x 4096 68 and 62, 2048 x 4096 x 4096 26 by 128
    //   1024 x 14336 x 4096: 39 and 45, 1152 x 14336 x 4096 67 and 47, 2048 x 8192 x 28672 253 and 332
    const auto tiles = [&](int64_t t) { return ((na + t - 1) / t) * ((nb + t - 1) / t); };
    const int64_t large = tiles(256), small = tiles(128), last = large % 256;
    const double by_large = double(large / 256) + (last ? 0.62 + 0.38 * double(last) / 256 : 0.0);
    p.tile = nblocks >= 16 && by_large <= 0.3 * double((small + 255) / 256) ? 256 : 128;
    p.a_tiles = int((na + p.tile - 1) / p.tile), p.b_tiles = int((nb + p.tile - 1) / p.tile);
    // Splits of the columns, as many as two workgroups a CU: the fastest by 0.95 us a stage of
    // one workgroup a CU, 1.2 of two, and 3 for the join and 0.6 for every MB of its sums. us
    //   65 x 4096 x 4096: none 15.3, two 13.1, four 11.7, eight 13.4; 512 x 4096 x 4096 13.7, 21.4, 22.4
    //   65 x 8192 x 28672: 94, 54, 41, 35; 256 x 8192 x 28672 115, 69, 61, 72
    p.splits = 1;
    double least = 0.0;
    for (int64_t n = 1; p.tile == 128 && n <= std::min<int64_t>(stages, 16) && (n == 1 || small * n <= 512); ++n) {
      const double us = double((stages + n - 1) / n) * (small * n <= 256 ? 0.95 : 1.2) +
                        (n > 1 ? 3.0 + 0.6e-6 * double(n * na * nb) * sizeof(float) : 0.0);
      if (n > 1 && us >= least) continue;
      least = us;
      p.splits = int(n);
    }
  }
  p.partial = p.splits > 1 ? align256(size_t(p.splits) * na * nb * sizeof(float)) : 0;
  return p;
}

// Bytes for up to kMaxRows rows of B.
size_t rows_bytes(int64_t na, int64_t nb, int64_t nblocks) {
  size_t need = plan(std::min(na, kMaxVecs), nb, nblocks).partial;
  if (na > kMaxVecs && na % kMaxVecs) need = std::max(need, plan(na % kMaxVecs, nb, nblocks).partial);
  return need;
}

hipError_t launch(const Mx4& a, const Mx4& b, void* d_y, int ytype, int64_t ldy, float* partial,
                  hipStream_t stream) {
  const Plan p = plan(a.nrows, b.nrows, b.nblocks);
  if (p.tile == 0) {
    auto go = [&](auto kern) {
      hipLaunchKernelGGL(kern, dim3(unsigned(p.b_tiles), unsigned(p.splits)), dim3(64 * p.waves), 0, stream,
                         a, b, p.splits, d_y, ytype, ldy, partial);
    };
    if (a.nrows <= 16) go(few_kernel<1>);
    else if (a.nrows <= 32) go(few_kernel<2>);
    else go(few_kernel<4>);
  } else {
    const int64_t units = (int64_t(p.b_tiles) * p.splits + 7) / 8 * 8;
    auto go = [&](auto kern, int waves) {
      hipLaunchKernelGGL(kern, dim3(unsigned(units * p.a_tiles)), dim3(64 * waves), size_t(4) * p.tile * (128 + 16),
                         stream, a, b, p.a_tiles, p.b_tiles, p.splits, d_y, ytype, ldy, partial);
    };
    const bool full = a.nrows >= p.tile && b.nrows >= p.tile && b.nblocks % kBlocks == 0 &&
                      b.row_words < int64_t(1) << 23;   // 64 rows are less than 2^32 bytes
    if (b.nblocks < 16) go(tile_kernel<2, 2, 2, 2, true, false>, 4);
    else if (p.tile == 256)
      full ? go(tile_kernel<4, 2, 2, 4, false, true>, 8) : go(tile_kernel<4, 2, 2, 4, false, false>, 8);
    else full ? go(tile_kernel<2, 2, 2, 2, false, true>, 4) : go(tile_kernel<2, 2, 2, 2, false, false>, 4);
  }
  if (p.splits > 1)
    launch_join(partial, p.splits, a.nrows, b.nrows, d_y, ytype, ldy, stream);
  return hipGetLastError();
}

}  // namespace

size_t mx4_matmul_workspace_bytes(int64_t na, int64_t nb, int64_t ncols) {
  const int64_t nblocks = (ncols + kMxBlock - 1) / kMxBlock;
  size_t need = rows_bytes(na, std::min(nb, kMaxRows), nblocks);
  if (nb > kMaxRows && nb % kMaxRows) need = std::max(need, rows_bytes(na, nb % kMaxRows, nblocks));
  return need;
}

hipError_t launch_mx4_matmul(const Mx4& a, const Mx4& b, void* d_y, int ytype, int64_t ldy, void* d_ws,
                             hipStream_t stream) {
  const int64_t size = ytype == SEEDQ_F32 ? 4 : 2;
  for (int64_t r = 0; r < b.nrows; r += kMaxRows)
    for (int64_t v = 0; v < a.nrows; v += kMaxVecs) {
      Mx4 rows = a.rows(v);
      rows.nrows = std::min(kMaxVecs, a.nrows - v);
      const hipError_t e = launch(rows, b.rows(r), static_cast<char*>(d_y) + (r + v * ldy) * size, ytype, ldy,
                                  static_cast<float*>(d_ws), stream);
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
}

}  // namespace seedq
