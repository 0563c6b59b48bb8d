// Declarations shared by the translation units of the operators of seedq_beam.h.
#pragma once

#include "seedq_beam.h"
#include "seedq_ops_internal.h"

namespace seedq {

struct BeamArgs {
  const void* logits;
  int64_t ld, batch, vocab;
  int beams, top;
  const float* scores;
  const uint8_t* finished;
  int64_t pad_token;
  float* score;
  int64_t *parent, *token;
};
size_t beam_select_workspace_bytes(int64_t batch, int beams, int64_t vocab, int top);
hipError_t launch_beam_select(const BeamArgs& a, int type, void* d_ws, hipStream_t stream);

hipError_t launch_beam_reorder(const seedq_beam_state* states, int64_t nstates, const int64_t* d_parent,
                               int64_t batch, int in_beams, int out_beams, hipStream_t stream);

}  // namespace seedq
