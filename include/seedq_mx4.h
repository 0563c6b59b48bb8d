/*
 * seedq_mx4.h -- operators of libseedq.so on matrices of microscaled 4-bit floats,
 * the 4-bit form that the matrix core multiplies itself: quantise, dequantise,
 * products with vectors in 16 or 32 bits, and products of two coded matrices.
 *
 * The conventions of seedq.h hold: d_* are device pointers of the current device,
 * the caller owns every buffer, work is enqueued asynchronously on hip_stream and
 * the library neither allocates memory nor synchronises. On an argument error
 * nothing is written and nothing is enqueued. Results do not depend on the stream
 * or on scheduling: every sum has a fixed order. The element types are those of
 * seedq_ops.h; buffers of a type are aligned to its size, rows may start anywhere a
 * leading dimension puts them.
 *
 * A matrix (nrows x ncols, ncols % 8 == 0, fewer than 2^31 blocks of 8, as in
 * seedq.h) is cut along each row into blocks of 32 columns, the last of which may be
 * short. The value of a code is
 *     w_hat = v 2^(e - 127),
 * e the block's biased exponent and v the code's 4-bit float: bit 3 the sign, the
 * magnitudes of the codes 0 .. 7 being 0, 0.5, 1, 1.5, 2, 3, 4, 6.
 *   codes: uint32 [nrows][seedq_mx4_row_words(ncols)], 16-byte aligned; column c of
 *          a row is the 4 bits from bit 4 (c % 8) of word c / 8. Rows are padded to
 *          16 bytes with zeros, which seedq_mx4_matmul relies on.
 *   scale: uint8 [nrows][ceil(ncols / 32)], the biased exponents; 255 makes every
 *          weight of the block NaN. 253 and 254, which the quantiser never writes,
 *          stand for weights past fp32's range, and what they enter may be infinite
 *          or NaN.
 */
#ifndef SEEDQ_MX4_H
#define SEEDQ_MX4_H

#include "seedq_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Words of a row of codes, 4 ceil(ncols / 32); 0 for a bad ncols. */
size_t seedq_mx4_row_words(int64_t ncols);

/*
 * Codes of W (type, row stride ldw >= ncols elements). With m the largest |w| of a
 * block, e = max(floor(log2 m) - 2, -127) + 127 (0 where m is 0), so that m lies below
 * 8 2^(e - 127); a code is w 2^(127 - e) rounded to the nearest of its values, of two
 * as near to the one of even code, above 6 to 6. The sign is kept, also of 0. A block
 * that holds a NaN or an infinity gets e = 255 and codes 0.
 * Asynchronous on hip_stream. Errors: SEEDQ_EINVAL, SEEDQ_EUNSUPPORTED (type),
 * SEEDQ_EHIP.
 */
int seedq_mx4_quantize(const void* d_W, int32_t type, int64_t ldw, int64_t nrows, int64_t ncols,
                       uint32_t* d_codes, uint8_t* d_scale, void* hip_stream);

/* W_hat (type, row stride ldw >= ncols elements) = v 2^(e - 127), rounded once: exact in
 * fp32 and bf16. Asynchronous on hip_stream. Errors as seedq_mx4_quantize. */
int seedq_mx4_dequantize(const uint32_t* d_codes, const uint8_t* d_scale, int64_t nrows,
                         int64_t ncols, void* d_W_hat, int32_t type, int64_t ldw, void* hip_stream);

/*
 * y_v = W_hat x_v for nvec >= 0 vectors, W_hat decoded on the fly and never stored.
 * The products are exact (but for bits of fp32 vectors below 2^-133), the sums held in
 * fp32, and y is rounded once.
 *   d_x: xtype [nvec][ncols], row stride ldx >= ncols elements.
 *   d_y: ytype [nvec][nrows], row stride ldy >= nrows elements; ytype is SEEDQ_F32
 *        or xtype. Not overlapping d_x.
 *   d_workspace: seedq_mx4_gemv_workspace_bytes(...) bytes, 256-byte aligned (may be
 *        NULL when that is 0).
 * A vector with a NaN or an infinity gives outputs that are not finite.
 * Asynchronous on hip_stream. Errors: SEEDQ_EINVAL, SEEDQ_EUNSUPPORTED (type),
 * SEEDQ_EWORKSPACE, SEEDQ_EHIP.
 */
size_t seedq_mx4_gemv_workspace_bytes(int64_t nrows, int64_t ncols, int64_t nvec, int32_t xtype);
int seedq_mx4_gemv(const uint32_t* d_codes, const uint8_t* d_scale, int64_t nrows, int64_t ncols,
                   int64_t nvec, const void* d_x, int32_t xtype, int64_t ldx, void* d_y,
                   int32_t ytype, int64_t ldy, void* d_workspace, size_t workspace_bytes,
                   void* hip_stream);

/*
 * Y = A_hat B_hat^T of two coded matrices of ncols columns, A of na >= 0 rows (the
 * vectors) and B of nb >= 1: Y[i][j] = sum_c A_hat[i][c] B_hat[j][c]. The matrix core
 * multiplies the codes; sums are held in fp32 and Y is rounded once.
 *   d_y: ytype [na][nb], row stride ldy >= nb elements, any of the three types.
 *   d_workspace: seedq_mx4_matmul_workspace_bytes(...) bytes, 256-byte aligned (may be
 *        NULL when that is 0).
 * Asynchronous on hip_stream. Errors: SEEDQ_EINVAL, SEEDQ_EUNSUPPORTED (type),
 * SEEDQ_EWORKSPACE, SEEDQ_EHIP.
 */
size_t seedq_mx4_matmul_workspace_bytes(int64_t na, int64_t nb, int64_t ncols);
int seedq_mx4_matmul(const uint32_t* d_a_codes, const uint8_t* d_a_scale, int64_t na,
                     const uint32_t* d_b_codes, const uint8_t* d_b_scale, int64_t nb, int64_t ncols,
                     void* d_y, int32_t ytype, int64_t ldy, void* d_workspace,
                     size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* SEEDQ_MX4_H */
