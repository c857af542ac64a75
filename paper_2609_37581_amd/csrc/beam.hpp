// Beam search's selection on the device: its arguments and launcher.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/trevs.h"

namespace trevs {

// Logits of a wave: 8 KB of them.
template <int BYTES>
constexpr int kBeamChunk = 8192 / BYTES;
inline int beam_chunk(int dtype) { return dtype == TREVS_BF16 ? kBeamChunk<2> : kBeamChunk<4>; }
constexpr int kBeamList = TREVS_MAX_BEAM_OUT + 16;
// Entries of a chunk's list: some more than are asked for, since it is not cut exactly.
inline int beam_stride(int n_out) { return n_out + 16; }

struct BeamArgs {
  const void* logits;
  long long ld;             // elements
  const float* score;
  const int32_t* done;
  float* score_out;
  int32_t* parent;
  int32_t* token;
  float2* part;             // [B,W,chunks] maximum and sum of exponentials
  uint64_t* cand;           // [B,W,chunks,stride] the chunk's best (key of the logit, complement of the token), in
                            // no order, 0: none
  int B, W, V, n, eos, chunks, stride;
};
hipError_t launch_beam_select(const BeamArgs& a, int dtype, hipStream_t s);

}  // namespace trevs
