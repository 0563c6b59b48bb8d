// Argument checks shared by the operators' C entry points.
#pragma once

#include <cstdint>

#include "seedq_ops_internal.h"

namespace seedq {

inline bool type_ok(int32_t t) { return t == SEEDQ_F32 || t == SEEDQ_F16 || t == SEEDQ_BF16; }
inline uintptr_t type_size(int32_t t) { return t == SEEDQ_F32 ? 4 : 2; }

inline bool misaligned(const void* p, uintptr_t to) {
  return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0;
}

// Leading dimensions and counts below keep every byte offset far inside 63 bits.
inline bool ld_ok(int64_t ld, int64_t n) { return ld >= n && ld <= (int64_t(1) << 40); }

inline bool shape_ok(int64_t nrows, int64_t ncols) {
  if (nrows <= 0 || ncols <= 0 || ncols % kC != 0) return false;
  const int64_t G = ncols / kC;
  return nrows <= (int64_t(1) << 31) / G && nrows * G < (int64_t(1) << 31);
}

inline bool logits_ok(int64_t nrows, int64_t vocab, int64_t ld) {
  return nrows >= 0 && nrows < (int64_t(1) << 31) && vocab >= 1 && vocab < (int64_t(1) << 31) &&
         ld_ok(ld, vocab);
}

inline int result(hipError_t e) { return e == hipSuccess ? SEEDQ_OK : SEEDQ_EHIP; }

}  // namespace seedq
