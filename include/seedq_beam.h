/*
 * seedq_beam.h -- beam search over the logits of a head, coded or not, by
 * libseedq.so: one step's selection over beams and vocabulary, and the states of the
 * beams moved to those that continue them.
 *
 * The conventions of seedq.h hold: d_* are device pointers of the current device,
 * the caller owns every buffer, work is enqueued asynchronously on hip_stream and
 * the library neither allocates memory nor synchronises. On an argument error
 * nothing is written and nothing is enqueued. Results do not depend on the stream
 * or on scheduling.
 */
#ifndef SEEDQ_BEAM_H
#define SEEDQ_BEAM_H

#include "seedq_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SEEDQ_MAX_BEAMS 32         /* beams of a sequence */
#define SEEDQ_MAX_BEAM_TOP 32      /* continuations of a sequence */
#define SEEDQ_MAX_BEAM_STATES 4096 /* tensors of one seedq_beam_reorder */

/*
 * The `top` (1 .. SEEDQ_MAX_BEAM_TOP) best continuations of each of batch >= 0
 * sequences, which have `beams` (1 .. SEEDQ_MAX_BEAMS) beams each. Beam b of a
 * sequence, whose score so far is s_b, offers every token v of its row x of logits with
 *     total = s_b + (x_v - log sum e^x),
 * exponentials and sums of two of them in fp32, the rest in fp64: the log of the sum errs by less
 * than 1.75e-7, and the total becomes fp32 once. A finished beam
 * offers pad_token alone, with total s_b. Continuations come by falling total, equal
 * totals by rising beam, equal ones of a beam by falling logit and rising token.
 *   d_logits: type [batch beams][vocab], row stride ld >= vocab; what lies between
 *        vocab and ld, and the rows of finished and dead beams, are not read.
 *   d_scores: fp32 [batch][beams]; -inf for a dead beam, which offers nothing.
 *   d_finished: uint8 [batch][beams], not 0 for a finished beam, or NULL.
 *   d_score (fp32, the totals), d_parent (int64, the beam in its sequence, 0 .. beams - 1)
 *   and d_token (int64): [batch][top].
 * Logits of -inf are no offers, and a row of nothing else offers nothing. Where fewer
 * than top are offered the rest is score -inf, parent -1, token -1. A sequence with a
 * score of NaN or +inf, or with a NaN or +inf in a row that is read, gets score NaN,
 * parent -1 and token -1 throughout.
 *   d_workspace: seedq_beam_select_workspace_bytes(...) bytes, 256-byte aligned.
 * Asynchronous on hip_stream. Errors: SEEDQ_EINVAL, SEEDQ_EUNSUPPORTED (type),
 * SEEDQ_EWORKSPACE, SEEDQ_EHIP.
 */
size_t seedq_beam_select_workspace_bytes(int64_t batch, int32_t beams, int64_t vocab, int32_t top);
int seedq_beam_select(const void* d_logits, int32_t type, int64_t ld, int64_t batch, int32_t beams,
                      int64_t vocab, const float* d_scores, const uint8_t* d_finished,
                      int64_t pad_token, int32_t top, float* d_score, int64_t* d_parent,
                      int64_t* d_token, void* d_workspace, size_t workspace_bytes,
                      void* hip_stream);

/*
 * A tensor of states: a row for each beam of each sequence, a row being `outer` pieces
 * of `inner` bytes each (a cache of heads x room x width of which a part is used: outer =
 * heads, inner = used x width). Strides are in bytes.
 */
typedef struct seedq_beam_state {
  const void* d_src;
  void* d_dst;
  int64_t src_row, dst_row;     /* from row to row */
  int64_t src_outer, dst_outer; /* from piece to piece */
  int64_t outer, inner;
} seedq_beam_state;

/*
 * Row (i, j) of every destination is row (i, parent[i][j]) of its source, for i < batch,
 * j < out_beams; sources have in_beams rows a sequence, destinations out_beams (both 1 ..
 * SEEDQ_MAX_BEAMS). A parent outside 0 .. in_beams - 1 gives zeros.
 *   states: host array of nstates (0 .. SEEDQ_MAX_BEAM_STATES), read before the call
 *        returns. Rows and pieces of a destination do not overlap each other.
 *   d_parent: int64 [batch][out_beams].
 * A destination may be its own source (d_dst == d_src, the same strides, out_beams ==
 * in_beams): rows that are their own parent are then neither read nor written. Otherwise
 * they do not overlap, and no destination overlaps another tensor of the call.
 * Asynchronous on hip_stream. Errors: SEEDQ_EINVAL, SEEDQ_EHIP.
 */
int seedq_beam_reorder(const seedq_beam_state* states, int64_t nstates, const int64_t* d_parent,
                       int64_t batch, int32_t in_beams, int32_t out_beams, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* SEEDQ_BEAM_H */
