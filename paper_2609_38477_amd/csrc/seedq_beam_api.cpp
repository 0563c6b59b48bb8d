// C ABI entry points of seedq_beam.h: argument checks and launches.
#include "seedq_beam_internal.h"
#include "seedq_ops_checks.h"

using namespace seedq;

namespace {

bool beams_ok(int64_t batch, int32_t beams) {
  return batch >= 0 && beams >= 1 && beams <= SEEDQ_MAX_BEAMS && batch < (int64_t(1) << 31) / beams;
}

// Strides and sizes of a piece; a row is at most 2^46 bytes.
bool bytes_ok(int64_t n) { return n >= 0 && n <= (int64_t(1) << 42); }

// Rows of `outer` pieces that do not overlap, in either order of the two.
bool apart(int64_t rows, int64_t row, int64_t outer, int64_t piece, int64_t inner) {
  typedef __int128 Wide;
  if (outer > 1 && piece < inner) return false;
  if (rows <= 1) return true;
  if (Wide(row) >= Wide(outer - 1) * piece + inner) return true;
  return outer > 1 && row >= inner && Wide(piece) >= Wide(rows - 1) * row + inner;
}

bool state_ok(const seedq_beam_state& s, int64_t rows_out, bool same) {
  if (s.outer < 0 || s.outer > (int64_t(1) << 31) || !bytes_ok(s.inner)) return false;
  if (s.outer == 0 || s.inner == 0) return true;
  if (!s.d_src || !s.d_dst || s.inner > (int64_t(1) << 46) / s.outer) return false;
  if (!bytes_ok(s.src_row) || !bytes_ok(s.dst_row) || !bytes_ok(s.src_outer) || !bytes_ok(s.dst_outer))
    return false;
  if (!apart(rows_out, s.dst_row, s.outer, s.dst_outer, s.inner)) return false;
  if (s.d_src == s.d_dst)
    return same && (rows_out == 1 || s.src_row == s.dst_row) && (s.outer == 1 || s.src_outer == s.dst_outer);
  return true;
}

}  // namespace

extern "C" {

size_t seedq_beam_select_workspace_bytes(int64_t batch, int32_t beams, int64_t vocab, int32_t top) {
  if (!beams_ok(batch, beams) || batch == 0 || !logits_ok(batch * beams, vocab, vocab) || top < 1 ||
      top > SEEDQ_MAX_BEAM_TOP)
    return 0;
  return beam_select_workspace_bytes(batch, beams, vocab, top);
}

int seedq_beam_select(const void* d_logits, int32_t type, int64_t ld, int64_t batch, int32_t beams,
                      int64_t vocab, const float* d_scores, const uint8_t* d_finished,
                      int64_t pad_token, int32_t top, float* d_score, int64_t* d_parent,
                      int64_t* d_token, void* d_workspace, size_t workspace_bytes,
                      void* hip_stream) {
  if (!type_ok(type)) return SEEDQ_EUNSUPPORTED;
  if (!beams_ok(batch, beams) || !logits_ok(batch * beams, vocab, ld) || top < 1 ||
      top > SEEDQ_MAX_BEAM_TOP || (d_finished && pad_token < 0))
    return SEEDQ_EINVAL;
  if (batch == 0) return SEEDQ_OK;
  if (!d_logits || !d_scores || !d_score || !d_parent || !d_token ||
      misaligned(d_logits, type_size(type)) || misaligned(d_scores, 4) || misaligned(d_score, 4) ||
      misaligned(d_parent, 8) || misaligned(d_token, 8))
    return SEEDQ_EINVAL;
  const size_t need = beam_select_workspace_bytes(batch, beams, vocab, top);
  if (!d_workspace || workspace_bytes < need || misaligned(d_workspace, 256)) return SEEDQ_EWORKSPACE;
  const BeamArgs a{d_logits, ld,         batch,     vocab,   beams,    top,
                   d_scores, d_finished, pad_token, d_score, d_parent, d_token};
  return result(launch_beam_select(a, type, d_workspace, static_cast<hipStream_t>(hip_stream)));
}

int seedq_beam_reorder(const seedq_beam_state* states, int64_t nstates, const int64_t* d_parent,
                       int64_t batch, int32_t in_beams, int32_t out_beams, void* hip_stream) {
  if (!beams_ok(batch, in_beams) || !beams_ok(batch, out_beams) || nstates < 0 ||
      nstates > SEEDQ_MAX_BEAM_STATES)
    return SEEDQ_EINVAL;
  if (batch == 0 || nstates == 0) return SEEDQ_OK;
  if (!states || !d_parent || misaligned(d_parent, 8)) return SEEDQ_EINVAL;
  for (int64_t i = 0; i < nstates; ++i)
    if (!state_ok(states[i], batch * out_beams, in_beams == out_beams))
      return SEEDQ_EINVAL;
  return result(launch_beam_reorder(states, nstates, d_parent, batch, in_beams, out_beams,
                                    static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
