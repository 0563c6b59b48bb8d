// C ABI entry points of seedq_mx4.h: argument checks and launches.
#include "seedq_mx4_internal.h"
#include "seedq_ops_checks.h"

using namespace seedq;

namespace {

int mx4_args(const uint32_t* d_codes, const uint8_t* d_scale, int64_t nrows, int64_t ncols, Mx4& q) {
  if (!d_codes || !d_scale || !shape_ok(nrows, ncols) || misaligned(d_codes, 16)) return SEEDQ_EINVAL;
  q = Mx4{d_codes, d_scale, nrows, ncols, q4_row_words(ncols), (ncols + kMxBlock - 1) / kMxBlock};
  return SEEDQ_OK;
}

}  // namespace

extern "C" {

size_t seedq_mx4_row_words(int64_t ncols) { return seedq_q4_row_words(ncols); }

int seedq_mx4_quantize(const void* d_W, int32_t type, int64_t ldw, int64_t nrows, int64_t ncols,
                       uint32_t* d_codes, uint8_t* d_scale, void* hip_stream) {
  if (!type_ok(type)) return SEEDQ_EUNSUPPORTED;
  Mx4 q;
  const int rc = mx4_args(d_codes, d_scale, nrows, ncols, q);
  if (rc != SEEDQ_OK) return rc;
  if (!d_W || misaligned(d_W, type_size(type)) || !ld_ok(ldw, ncols)) return SEEDQ_EINVAL;
  return result(launch_mx4_quantize(d_W, type, ldw, q, static_cast<hipStream_t>(hip_stream)));
}

int seedq_mx4_dequantize(const uint32_t* d_codes, const uint8_t* d_scale, int64_t nrows,
                         int64_t ncols, void* d_W_hat, int32_t type, int64_t ldw, void* hip_stream) {
  if (!type_ok(type)) return SEEDQ_EUNSUPPORTED;
  Mx4 q;
  const int rc = mx4_args(d_codes, d_scale, nrows, ncols, q);
  if (rc != SEEDQ_OK) return rc;
  if (!d_W_hat || misaligned(d_W_hat, type_size(type)) || !ld_ok(ldw, ncols)) return SEEDQ_EINVAL;
  return result(launch_mx4_dequantize(q, d_W_hat, type, ldw, static_cast<hipStream_t>(hip_stream)));
}

size_t seedq_mx4_gemv_workspace_bytes(int64_t nrows, int64_t ncols, int64_t nvec, int32_t xtype) {
  if (!shape_ok(nrows, ncols) || nvec <= 0 || nvec > (int64_t(1) << 24) || !type_ok(xtype)) return 0;
  return mx4_gemv_workspace_bytes(nrows, ncols, nvec, xtype);
}

int seedq_mx4_gemv(const uint32_t* d_codes, const uint8_t* d_scale, int64_t nrows, int64_t ncols,
                   int64_t nvec, const void* d_x, int32_t xtype, int64_t ldx, void* d_y,
                   int32_t ytype, int64_t ldy, void* d_workspace, size_t workspace_bytes,
                   void* hip_stream) {
  if (!type_ok(xtype) || !type_ok(ytype) || (ytype != SEEDQ_F32 && ytype != xtype))
    return SEEDQ_EUNSUPPORTED;
  Mx4 q;
  const int rc = mx4_args(d_codes, d_scale, nrows, ncols, q);
  if (rc != SEEDQ_OK) return rc;
  if (nvec < 0 || nvec > (int64_t(1) << 24)) return SEEDQ_EINVAL;
  if (nvec == 0) return SEEDQ_OK;
  if (!d_x || !d_y || misaligned(d_x, type_size(xtype)) || misaligned(d_y, type_size(ytype)) ||
      !ld_ok(ldx, ncols) || !ld_ok(ldy, nrows))
    return SEEDQ_EINVAL;
  const size_t need = mx4_gemv_workspace_bytes(nrows, ncols, nvec, xtype);
  if (need && (!d_workspace || workspace_bytes < need || misaligned(d_workspace, 256)))
    return SEEDQ_EWORKSPACE;
  return result(launch_mx4_gemv(q, nvec, d_x, xtype, ldx, d_y, ytype, ldy, d_workspace,
                                static_cast<hipStream_t>(hip_stream)));
}

size_t seedq_mx4_matmul_workspace_bytes(int64_t na, int64_t nb, int64_t ncols) {
  if (!shape_ok(na, ncols) || !shape_ok(nb, ncols)) return 0;
  return mx4_matmul_workspace_bytes(na, nb, ncols);
}

int seedq_mx4_matmul(const uint32_t* d_a_codes, const uint8_t* d_a_scale, int64_t na,
                     const uint32_t* d_b_codes, const uint8_t* d_b_scale, int64_t nb, int64_t ncols,
                     void* d_y, int32_t ytype, int64_t ldy, void* d_workspace,
                     size_t workspace_bytes, void* hip_stream) {
  if (!type_ok(ytype)) return SEEDQ_EUNSUPPORTED;
  Mx4 a, b;
  int rc = mx4_args(d_b_codes, d_b_scale, nb, ncols, b);
  if (rc != SEEDQ_OK) return rc;
  if (na == 0) return SEEDQ_OK;
  rc = mx4_args(d_a_codes, d_a_scale, na, ncols, a);
  if (rc != SEEDQ_OK) return rc;
  if (!d_y || misaligned(d_y, type_size(ytype)) || !ld_ok(ldy, nb)) return SEEDQ_EINVAL;
  const size_t need = mx4_matmul_workspace_bytes(na, nb, ncols);
  if (need && (!d_workspace || workspace_bytes < need || misaligned(d_workspace, 256)))
    return SEEDQ_EWORKSPACE;
  return result(launch_mx4_matmul(a, b, d_y, ytype, ldy, d_workspace,
                                  static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
