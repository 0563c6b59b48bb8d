// Declarations shared by the translation units of the operators of seedq_ops.h.
#pragma once

#include "seedq_internal.h"
#include "seedq_ops.h"

namespace seedq {

inline int64_t q4_row_words(int64_t ncols) { return 4 * ((ncols + 31) / 32); }
inline int64_t q4_groups(int64_t ncols, int group) { return (ncols + group - 1) / group; }

// Rows of one launch: a grid has fewer than 2^32 threads along a dimension.
constexpr int64_t kMaxRows = int64_t(1) << 21;

// A matrix in 4 bits. gshift = log2(group); zero may be null.
struct Q4 {
  const uint32_t* codes;
  const uint16_t* scale;
  const uint8_t* zero;
  int64_t nrows, ncols, row_words, ngroups;
  int gshift;
  // Up to kMaxRows rows from row r on.
  Q4 rows(int64_t r) const {
    Q4 q = *this;
    q.codes += r * row_words;
    q.scale += r * ngroups;
    if (zero) q.zero += r * ngroups;
    q.nrows = nrows - r < kMaxRows ? nrows - r : kMaxRows;
    return q;
  }
};

// q's arrays are written.
hipError_t launch_q4_quantize(const void* d_W, int type, int64_t ldw, const Q4& q,
                              hipStream_t stream);
hipError_t launch_q4_dequantize(const Q4& q, void* d_W_hat, int type, int64_t ldw,
                                hipStream_t stream);
size_t q4_gemv_workspace_bytes(int64_t nrows, int64_t ncols, int64_t nvec, int xtype);
hipError_t launch_q4_gemv(const Q4& q, int64_t nvec, const void* d_x, int xtype, int64_t ldx,
                          void* d_y, int ytype, int64_t ldy, void* d_ws, hipStream_t stream);

struct LogprobArgs {
  const void* logits;
  int64_t ld, nrows, vocab;
  const int64_t* tokens;
  int top;
  float *logprob, *entropy, *lse;
  int64_t* top_token;
  float* top_logprob;
};
size_t token_logprobs_workspace_bytes(int64_t nrows, int64_t vocab, int top);
hipError_t launch_token_logprobs(const LogprobArgs& a, int type, void* d_ws, hipStream_t stream);

struct LogprobGradArgs {
  const void* logits;
  int64_t ld, nrows, vocab;
  const int64_t* tokens;
  const float *lse, *entropy, *g, *h;
  void* grad;
  int64_t ldg;
};
hipError_t launch_token_logprobs_backward(const LogprobGradArgs& a, int type, hipStream_t stream);

}  // namespace seedq
