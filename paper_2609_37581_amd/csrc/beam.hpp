// Beam search's selection on the device: its arguments and launcher.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/trevs.h"

namespace trevs {

constexpr int kBeamChunk = 8192;  // logits of a workgroup

struct BeamArgs {
  const void* logits;
  long long ld;             // elements
  const float* score;
  const int32_t* done;
  float* score_out;
  int32_t* parent;
  int32_t* token;
  float2* part;             // [B,W,chunks] maximum and sum of exponentials
  uint64_t* cand;           // [B,W,chunks,n] the chunk's best (key of the logit, complement of the token), 0: none
  int B, W, V, n, eos, chunks;
};
hipError_t launch_beam_select(const BeamArgs& a, int dtype, hipStream_t s);

}  // namespace trevs
