/*
 * seedq_ops.h -- operators of libseedq.so beside the seed codec of seedq.h:
 *
 * - weights in 4 bits with a scale for each group of columns, the ordinary format
 *   that the codec's comparisons are made against: quantise, dequantise, and
 *   products straight from the codes for one vector, a batch or a prompt;
 * - what a coded head or layer is judged by: log probabilities of given tokens
 *   (perplexity), the entropy, the top alternatives, and their gradient at the
 *   logits (the measured counterpart of the data-free gradient size rho).
 *
 * The conventions of seedq.h hold: d_* are device pointers of the current device,
 * the caller owns every buffer, work is enqueued asynchronously on hip_stream and
 * the library neither allocates memory nor synchronises. On an argument error
 * nothing is written and nothing is enqueued. Results do not depend on the stream
 * or on scheduling: every sum has a fixed order.
 *
 * Element types of the arguments called *type. Buffers of a type are aligned to
 * its size; rows may start anywhere a leading dimension puts them.
 */
#ifndef SEEDQ_OPS_H
#define SEEDQ_OPS_H

#include "seedq.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SEEDQ_F32 0
#define SEEDQ_F16 1
#define SEEDQ_BF16 2

#define SEEDQ_MAX_TOP 32        /* alternatives of seedq_token_logprobs */

/*
 * ---- 4-bit weights with group scales.
 *
 * W (nrows x ncols, ncols % 8 == 0, fewer than 2^31 blocks of 8, as in seedq.h) is
 * cut along each row into groups of `group` columns (32, 64, 128, 256 or 512; the
 * last group of a row may be short). The value of a code u in 0 .. 15 is
 *     w_hat = s (u - z),
 * s the group's fp16 scale and z its zero point, or 8 where there are none; the
 * product is exact in fp32.
 *   codes: uint32 [nrows][seedq_q4_row_words(ncols)], 16-byte aligned; column c of
 *          a row is the 4 bits from bit 4 (c % 8) of word c / 8. Rows are padded to
 *          16 bytes with zeros, which no call reads as weights.
 *   scale: fp16 [nrows][ngroups], ngroups = ceil(ncols / group).
 *   zero:  uint8 [nrows][ngroups], 0 .. 15 (the low 4 bits are read), or NULL.
 */

/* Words of a row of codes, 4 ceil(ncols / 32); 0 for a bad ncols. */
size_t seedq_q4_row_words(int64_t ncols);

/*
 * Round-to-nearest codes of W (finite; type, row stride ldw >= ncols elements).
 * Without zero points (d_zero NULL):
 *     s = fp16(fl32(max |w| / 7)),        u = 8 + clamp(rne(fl32(w / s)), -8, 7);
 * with them, lo = min(0, min w) and hi = max(0, max w) over the group:
 *     s = fp16(fl32(fl32(hi - lo) / 15)), z = clamp(rne(fl32(-lo / s)), 0, 15),
 *     u = clamp(rne(fl32(w / s)) + z, 0, 15).
 * fl32 and fp16 round to nearest even; s is at most 65504; where s is 0 every code
 * stands for 0. A group that holds a NaN or an infinity gets a NaN scale (its
 * weights decode to NaN).
 * Asynchronous on hip_stream. Errors: SEEDQ_EINVAL, SEEDQ_EUNSUPPORTED (group or
 * type), SEEDQ_EHIP.
 */
int seedq_q4_quantize(const void* d_W, int32_t type, int64_t ldw, int64_t nrows, int64_t ncols,
                      int32_t group, uint32_t* d_codes, void* d_scale, uint8_t* d_zero,
                      void* hip_stream);

/* W_hat (type, row stride ldw >= ncols elements) = s (u - z), rounded once.
 * Asynchronous on hip_stream. Errors as seedq_q4_quantize. */
int seedq_q4_dequantize(const uint32_t* d_codes, const void* d_scale, const uint8_t* d_zero,
                        int64_t nrows, int64_t ncols, int32_t group, void* d_W_hat, int32_t type,
                        int64_t ldw, void* hip_stream);

/*
 * y_v = W_hat x_v for nvec >= 0 vectors, W_hat decoded on the fly and never stored.
 * The products and sums are held in fp32 and y is rounded once.
 *   d_x: xtype [nvec][ncols], row stride ldx >= ncols elements.
 *   d_y: ytype [nvec][nrows], row stride ldy >= nrows elements; ytype is SEEDQ_F32
 *        or xtype. Not overlapping d_x.
 *   d_workspace: seedq_q4_gemv_workspace_bytes(...) bytes, 256-byte aligned (may be
 *        NULL when that is 0).
 * They pass the range of fp32 only where sums of s (u - z) x do.
 * A vector with a NaN or an infinity gives outputs that are not finite.
 * Asynchronous on hip_stream. Errors: SEEDQ_EINVAL, SEEDQ_EUNSUPPORTED (group or
 * type), SEEDQ_EWORKSPACE, SEEDQ_EHIP.
 */
size_t seedq_q4_gemv_workspace_bytes(int64_t nrows, int64_t ncols, int64_t nvec, int32_t xtype);
int seedq_q4_gemv(const uint32_t* d_codes, const void* d_scale, const uint8_t* d_zero,
                  int64_t nrows, int64_t ncols, int32_t group, int64_t nvec, const void* d_x,
                  int32_t xtype, int64_t ldx, void* d_y, int32_t ytype, int64_t ldy,
                  void* d_workspace, size_t workspace_bytes, void* hip_stream);

/*
 * ---- Log probabilities of given tokens.
 *
 * For each of nrows >= 0 rows x of logits (type, vocab >= 1 entries, row stride ld >=
 * vocab elements; what lies between vocab and ld is not read), with m = max x and
 * S = sum e^(x - m), in fp32 or wider:
 *   d_lse[t]     = m + log S;
 *   d_logprob[t] = x[token] - lse, the token from d_tokens (int64 [nrows]). A
 *                  negative token asks for nothing: 0. A token >= vocab: NaN;
 *   d_entropy[t] = -sum p log p = log S - sum e^(x - m) (x - m) / S, in nats;
 *   d_top_token, d_top_logprob [nrows][top]: the `top` (0 .. SEEDQ_MAX_TOP) largest
 *                  logits in falling order, equal ones by rising token, and their
 *                  log probabilities. Logits of -inf are no alternatives: where
 *                  fewer are left the rest is token -1, log probability -inf.
 * A logit of -inf has probability 0. A row of nothing else has lse -inf, log
 * probability -inf, entropy 0 and no alternatives. A row with a NaN or +inf gives
 * NaN (0 for a negative token) and tokens -1.
 *   d_logprob, d_entropy, d_lse: fp32 [nrows], each nullable (d_logprob needs
 *   d_tokens); d_top_token (int64) and d_top_logprob (fp32): NULL iff top == 0.
 *   d_workspace: seedq_token_logprobs_workspace_bytes(...) bytes, 256-byte aligned
 *   (may be NULL when that is 0).
 * Asynchronous on hip_stream. Errors: SEEDQ_EINVAL, SEEDQ_EUNSUPPORTED (type),
 * SEEDQ_EWORKSPACE, SEEDQ_EHIP.
 */
size_t seedq_token_logprobs_workspace_bytes(int64_t nrows, int64_t vocab, int32_t top);
int seedq_token_logprobs(const void* d_logits, int32_t type, int64_t ld, int64_t nrows,
                         int64_t vocab, const int64_t* d_tokens, int32_t top, float* d_logprob,
                         float* d_entropy, float* d_lse, int64_t* d_top_token,
                         float* d_top_logprob, void* d_workspace, size_t workspace_bytes,
                         void* hip_stream);

/*
 * Gradient of sum_t (g_t logprob_t + h_t entropy_t) at the logits, from the lse and
 * entropy that seedq_token_logprobs gave:
 *   dx_v = g (1[v = token] - p_v) - h p_v (log p_v + entropy),  p_v = e^(x_v - lse),
 * rounded once to the logits' type. Where |lse| >= 1024, which fp32 holds too coarsely
 * for p (a row of nothing but the type's lowest value: log S is lost), p is taken from
 * the row's own m and S, at the price of a second pass over it. p is 0 at -inf (the
 * gradient there is g at the token itself, else 0). A row without any finite logit (lse -inf) has gradient 0;
 * a NaN lse gives NaN. A negative token has no log probability to differentiate; one
 * >= vocab gives a NaN row, without a finite logit too. Without g the tokens play no
 * part.
 *   d_grad_logprob (g), d_grad_entropy (h): fp32 [nrows], at least one not NULL;
 *   d_grad_logprob needs d_tokens, d_grad_entropy needs d_entropy.
 *   d_grad_logits: type [nrows][vocab], row stride ldg >= vocab elements; nothing
 *   past vocab is written. It may be d_logits itself when ldg == ld.
 * Asynchronous on hip_stream. Errors: SEEDQ_EINVAL, SEEDQ_EUNSUPPORTED (type),
 * SEEDQ_EHIP.
 */
int seedq_token_logprobs_backward(const void* d_logits, int32_t type, int64_t ld, int64_t nrows,
                                  int64_t vocab, const int64_t* d_tokens, const float* d_lse,
                                  const float* d_entropy, const float* d_grad_logprob,
                                  const float* d_grad_entropy, void* d_grad_logits, int64_t ldg,
                                  void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* SEEDQ_OPS_H */
