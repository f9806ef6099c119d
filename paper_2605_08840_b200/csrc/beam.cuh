// Selection of the best continuations of a request's hypotheses: what the entry point hands to the kernels.
#pragma once

#include "restkv_common.cuh"

namespace restkv {

constexpr int kBeamsPerRequest = 64, kBeamOut = 64;   // at most

struct BeamProblem {
  int batch, beams, vocab, n_out;
  bool f32;
  long long stride;            // elements between rows of logits
  int pad_token;
  const void* logits;
  const float* scores;
  const uint8_t* finished;     // or null
  int *parents, *tokens;
  float* scores_out;
};

size_t beam_bytes(const BeamProblem& p, int sm_count);
cudaError_t launch_beam_select(const BeamProblem& p, int sm_count, void* workspace, cudaStream_t st);

}  // namespace restkv
