// Host interface of beam.hip: a step of beam search. All arguments are validated by
// the caller.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "head_types.h"

namespace w2v {

struct BeamArgs {
  const void* logits;  // (batch * beams) x V, stride ld
  int64_t ld;
  int32_t batch, beams, V, dtype, width, end;
  const float* scores;      // [batch][beams]
  const uint8_t* finished;  // [batch][beams] or NULL
  int32_t* words;           // [batch][width] each
  int32_t* parents;
  float* new_scores;
  uint8_t* new_finished;  // or NULL
};

size_t beam_workspace_bytes(int32_t batch, int32_t beams, int32_t width, int32_t V,
                            int32_t dtype);
hipError_t launch_beam_step(const BeamArgs& a, void* workspace, hipStream_t s);

struct ReorderArgs {
  w2v_beam_state states[W2V_MAX_BEAM_STATES];
  const int32_t* parents;  // [batch][width]
  int32_t count, batch, beams, width;
  int32_t* status;
  Divisor by_row[W2V_MAX_BEAM_STATES];  // a row's chunks; set by the launch
};
hipError_t launch_beam_reorder(const ReorderArgs& a, hipStream_t s);

}  // namespace w2v
