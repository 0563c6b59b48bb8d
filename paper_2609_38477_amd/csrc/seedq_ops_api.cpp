// C ABI entry points of seedq_ops.h: argument checks and launches.
#include "seedq_ops_internal.h"

using namespace seedq;

namespace {

bool type_ok(int32_t t) { return t == SEEDQ_F32 || t == SEEDQ_F16 || t == SEEDQ_BF16; }
uintptr_t type_size(int32_t t) { return t == SEEDQ_F32 ? 4 : 2; }

bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// Leading dimensions and counts below keep every byte offset far inside 63 bits.
bool ld_ok(int64_t ld, int64_t n) { return ld >= n && ld <= (int64_t(1) << 40); }

int group_shift(int32_t group) {
  for (int s = 5; s <= 9; ++s)
    if (group == 1 << s) return s;
  return 0;
}

bool shape_ok(int64_t nrows, int64_t ncols) {
  if (nrows <= 0 || ncols <= 0 || ncols % kC != 0) return false;
  const int64_t G = ncols / kC;
  return nrows <= (int64_t(1) << 31) / G && nrows * G < (int64_t(1) << 31);
}

int q4_args(const uint32_t* d_codes, const void* d_scale, const uint8_t* d_zero, int64_t nrows,
            int64_t ncols, int32_t group, Q4& q) {
  if (!d_codes || !d_scale || !shape_ok(nrows, ncols)) return SEEDQ_EINVAL;
  if (misaligned(d_codes, 16) || misaligned(d_scale, 2)) return SEEDQ_EINVAL;
  const int gshift = group_shift(group);
  if (!gshift) return SEEDQ_EUNSUPPORTED;
  q = Q4{d_codes, static_cast<const uint16_t*>(d_scale), d_zero, nrows, ncols, q4_row_words(ncols),
         q4_groups(ncols, group), gshift};
  return SEEDQ_OK;
}

int result(hipError_t e) { return e == hipSuccess ? SEEDQ_OK : SEEDQ_EHIP; }

}  // namespace

extern "C" {

size_t seedq_q4_row_words(int64_t ncols) {
  return ncols > 0 && ncols % kC == 0 && ncols / kC < (int64_t(1) << 31) ? size_t(q4_row_words(ncols))
                                                                        : 0;
}

int seedq_q4_quantize(const void* d_W, int32_t type, int64_t ldw, int64_t nrows, int64_t ncols,
                      int32_t group, uint32_t* d_codes, void* d_scale, uint8_t* d_zero,
                      void* hip_stream) {
  if (!type_ok(type)) return SEEDQ_EUNSUPPORTED;
  Q4 q;
  const int rc = q4_args(d_codes, d_scale, d_zero, nrows, ncols, group, q);
  if (rc != SEEDQ_OK) return rc;
  if (!d_W || misaligned(d_W, type_size(type)) || !ld_ok(ldw, ncols)) return SEEDQ_EINVAL;
  return result(launch_q4_quantize(d_W, type, ldw, q, static_cast<hipStream_t>(hip_stream)));
}

int seedq_q4_dequantize(const uint32_t* d_codes, const void* d_scale, const uint8_t* d_zero,
                        int64_t nrows, int64_t ncols, int32_t group, void* d_W_hat, int32_t type,
                        int64_t ldw, void* hip_stream) {
  if (!type_ok(type)) return SEEDQ_EUNSUPPORTED;
  Q4 q;
  const int rc = q4_args(d_codes, d_scale, d_zero, nrows, ncols, group, q);
  if (rc != SEEDQ_OK) return rc;
  if (!d_W_hat || misaligned(d_W_hat, type_size(type)) || !ld_ok(ldw, ncols)) return SEEDQ_EINVAL;
  return result(launch_q4_dequantize(q, d_W_hat, type, ldw, static_cast<hipStream_t>(hip_stream)));
}

size_t seedq_q4_gemv_workspace_bytes(int64_t nrows, int64_t ncols, int64_t nvec, int32_t xtype) {
  if (!shape_ok(nrows, ncols) || nvec <= 0 || nvec > (int64_t(1) << 24) || !type_ok(xtype)) return 0;
  return q4_gemv_workspace_bytes(nrows, ncols, nvec, xtype);
}

int seedq_q4_gemv(const uint32_t* d_codes, const void* d_scale, const uint8_t* d_zero,
                  int64_t nrows, int64_t ncols, int32_t group, int64_t nvec, const void* d_x,
                  int32_t xtype, int64_t ldx, void* d_y, int32_t ytype, int64_t ldy,
                  void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  if (!type_ok(xtype) || !type_ok(ytype) || (ytype != SEEDQ_F32 && ytype != xtype))
    return SEEDQ_EUNSUPPORTED;
  Q4 q;
  const int rc = q4_args(d_codes, d_scale, d_zero, nrows, ncols, group, q);
  if (rc != SEEDQ_OK) return rc;
  if (nvec < 0 || nvec > (int64_t(1) << 24)) return SEEDQ_EINVAL;
  if (nvec == 0) return SEEDQ_OK;
  if (!d_x || !d_y || misaligned(d_x, type_size(xtype)) || misaligned(d_y, type_size(ytype)) ||
      !ld_ok(ldx, ncols) || !ld_ok(ldy, nrows))
    return SEEDQ_EINVAL;
  const size_t need = q4_gemv_workspace_bytes(nrows, ncols, nvec, xtype);
  if (need && (!d_workspace || workspace_bytes < need || misaligned(d_workspace, 256)))
    return SEEDQ_EWORKSPACE;
  return result(launch_q4_gemv(q, nvec, d_x, xtype, ldx, d_y, ytype, ldy, d_workspace,
                               static_cast<hipStream_t>(hip_stream)));
}

namespace {

bool logits_ok(int64_t nrows, int64_t vocab, int64_t ld) {
  return nrows >= 0 && nrows < (int64_t(1) << 31) && vocab >= 1 && vocab < (int64_t(1) << 31) &&
         ld_ok(ld, vocab);
}

}  // namespace

size_t seedq_token_logprobs_workspace_bytes(int64_t nrows, int64_t vocab, int32_t top) {
  if (nrows <= 0 || !logits_ok(nrows, vocab, vocab) || top < 0 || top > SEEDQ_MAX_TOP) return 0;
  return token_logprobs_workspace_bytes(nrows, vocab, top);
}

int seedq_token_logprobs(const void* d_logits, int32_t type, int64_t ld, int64_t nrows,
                         int64_t vocab, const int64_t* d_tokens, int32_t top, float* d_logprob,
                         float* d_entropy, float* d_lse, int64_t* d_top_token,
                         float* d_top_logprob, void* d_workspace, size_t workspace_bytes,
                         void* hip_stream) {
  if (!type_ok(type)) return SEEDQ_EUNSUPPORTED;
  if (!logits_ok(nrows, vocab, ld) || top < 0 || top > SEEDQ_MAX_TOP) return SEEDQ_EINVAL;
  if (nrows == 0) return SEEDQ_OK;
  if ((top > 0) != (d_top_token != nullptr) || (top > 0) != (d_top_logprob != nullptr))
    return SEEDQ_EINVAL;
  if ((d_logprob && !d_tokens) || (!d_logprob && !d_entropy && !d_lse && top == 0))
    return SEEDQ_EINVAL;
  if (!d_logits || misaligned(d_logits, type_size(type)) || misaligned(d_tokens, 8) ||
      misaligned(d_logprob, 4) || misaligned(d_entropy, 4) || misaligned(d_lse, 4) ||
      misaligned(d_top_token, 8) || misaligned(d_top_logprob, 4))
    return SEEDQ_EINVAL;
  const size_t need = token_logprobs_workspace_bytes(nrows, vocab, top);
  if (need && (!d_workspace || workspace_bytes < need || misaligned(d_workspace, 256)))
    return SEEDQ_EWORKSPACE;
  const LogprobArgs a{d_logits, ld,        nrows, vocab,       d_tokens,     top,
                      d_logprob, d_entropy, d_lse, d_top_token, d_top_logprob};
  return result(launch_token_logprobs(a, type, d_workspace, static_cast<hipStream_t>(hip_stream)));
}

int seedq_token_logprobs_backward(const void* d_logits, int32_t type, int64_t ld, int64_t nrows,
                                  int64_t vocab, const int64_t* d_tokens, const float* d_lse,
                                  const float* d_entropy, const float* d_grad_logprob,
                                  const float* d_grad_entropy, void* d_grad_logits, int64_t ldg,
                                  void* hip_stream) {
  if (!type_ok(type)) return SEEDQ_EUNSUPPORTED;
  if (!logits_ok(nrows, vocab, ld) || !ld_ok(ldg, vocab)) return SEEDQ_EINVAL;
  if (nrows == 0) return SEEDQ_OK;
  if (!d_grad_logprob && !d_grad_entropy) return SEEDQ_EINVAL;
  if ((d_grad_logprob && !d_tokens) || (d_grad_entropy && !d_entropy)) return SEEDQ_EINVAL;
  if (d_grad_logits && d_grad_logits == d_logits && ldg != ld) return SEEDQ_EINVAL;
  if (!d_logits || !d_lse || !d_grad_logits || misaligned(d_logits, type_size(type)) ||
      misaligned(d_grad_logits, type_size(type)) || misaligned(d_tokens, 8) ||
      misaligned(d_lse, 4) || misaligned(d_entropy, 4) || misaligned(d_grad_logprob, 4) ||
      misaligned(d_grad_entropy, 4))
    return SEEDQ_EINVAL;
  const LogprobGradArgs a{d_logits,  ld,             nrows,          vocab,         d_tokens, d_lse,
                          d_entropy, d_grad_logprob, d_grad_entropy, d_grad_logits, ldg};
  return result(launch_token_logprobs_backward(a, type, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
