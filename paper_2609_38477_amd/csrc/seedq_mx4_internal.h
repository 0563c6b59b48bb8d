// Declarations shared by the translation units of the operators of seedq_mx4.h.
#pragma once

#include "seedq_mx4.h"
#include "seedq_ops_internal.h"

namespace seedq {

constexpr int kMxBlock = 32;

// A matrix of microscaled 4-bit floats; rows are padded to whole blocks of 16 bytes.
struct Mx4 {
  const uint32_t* codes;
  const uint8_t* scale;
  int64_t nrows, ncols, row_words, nblocks;
  // Up to kMaxRows rows from row r on.
  Mx4 rows(int64_t r) const {
    Mx4 q = *this;
    q.codes += r * row_words;
    q.scale += r * nblocks;
    q.nrows = nrows - r < kMaxRows ? nrows - r : kMaxRows;
    return q;
  }
};

// q's arrays are written.
hipError_t launch_mx4_quantize(const void* d_W, int type, int64_t ldw, const Mx4& q,
                               hipStream_t stream);
hipError_t launch_mx4_dequantize(const Mx4& q, void* d_W_hat, int type, int64_t ldw,
                                 hipStream_t stream);
size_t mx4_gemv_workspace_bytes(int64_t nrows, int64_t ncols, int64_t nvec, int xtype);
hipError_t launch_mx4_gemv(const Mx4& q, int64_t nvec, const void* d_x, int xtype, int64_t ldx,
                           void* d_y, int ytype, int64_t ldy, void* d_ws, hipStream_t stream);
size_t mx4_matmul_workspace_bytes(int64_t na, int64_t nb, int64_t ncols);
hipError_t launch_mx4_matmul(const Mx4& a, const Mx4& b, void* d_y, int ytype, int64_t ldy, void* d_ws,
                             hipStream_t stream);

}  // namespace seedq
