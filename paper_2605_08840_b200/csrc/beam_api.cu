// C ABI of the selection over hypotheses: argument checks and the launch.
#include "beam.cuh"
#include "restkv_handle.cuh"

namespace restkv {

static restkv_status make_beams(const restkv_beams* s, BeamProblem* out) {
  if (!s) return RESTKV_ERR_INVALID_ARG;
  if (s->batch < 1 || s->beams < 1 || s->vocab < 1 || s->n_out < 1) return RESTKV_ERR_INVALID_ARG;
  if (s->dtype != RESTKV_BF16 && s->dtype != RESTKV_F32) return RESTKV_ERR_INVALID_ARG;
  if (s->stride != 0 && s->stride < s->vocab) return RESTKV_ERR_INVALID_ARG;
  if (s->beams > kBeamsPerRequest || s->n_out > kBeamOut) return RESTKV_ERR_UNSUPPORTED;
  if (s->vocab > 0x40000000) return RESTKV_ERR_UNSUPPORTED;   // places in a row, rounded up to a block's share, are counted in 32 bits
  BeamProblem p{};
  p.batch = s->batch; p.beams = s->beams; p.vocab = s->vocab; p.n_out = s->n_out;
  p.f32 = s->dtype == RESTKV_F32;
  p.stride = s->stride ? s->stride : s->vocab;
  p.pad_token = s->pad_token;
  // a block per 2048 tokens of a row at most, all in one grid
  if ((long long)p.batch * p.beams > 0x7FFFFFFFll / (p.vocab / 2048 + 2)) return RESTKV_ERR_UNSUPPORTED;
  *out = p;
  return RESTKV_OK;
}

static int current_sms() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && sms > 0)
    return sms;
  (void)cudaGetLastError();
  return 148;
}

}  // namespace restkv

using namespace restkv;

extern "C" {

size_t restkv_beam_workspace_bytes(const restkv_beams* beams) {
  BeamProblem p;
  if (make_beams(beams, &p) != RESTKV_OK) return 0;
  return align256(beam_bytes(p, current_sms()));
}

restkv_status restkv_beam_select(restkv_handle* h, const restkv_beams* beams, const void* logits, const float* scores, const uint8_t* finished,
                                 int32_t* parents, int32_t* tokens, float* scores_out, void* workspace, size_t workspace_bytes,
                                 restkv_stream stream) {
  if (!h || !logits || !scores || !parents || !tokens || !scores_out) return RESTKV_ERR_INVALID_ARG;
  if (!aligned16(logits)) return RESTKV_ERR_INVALID_ARG;
  BeamProblem p;
  const restkv_status s = make_beams(beams, &p);
  if (s != RESTKV_OK) return s;
  if (!workspace || ((uintptr_t)workspace & 255u) != 0 || workspace_bytes < align256(beam_bytes(p, h->sm_count))) return RESTKV_ERR_WORKSPACE;
  if (!on_device(h)) return RESTKV_ERR_INVALID_ARG;
  p.logits = logits; p.scores = scores; p.finished = finished;
  p.parents = parents; p.tokens = tokens; p.scores_out = scores_out;
  Call call{h, (cudaStream_t)stream};
  RESTKV_LAUNCH(call, RESTKV_KERNEL_NONE, launch_beam_select(p, h->sm_count, workspace, call.st), 2);
  return RESTKV_OK;
}

}  // extern "C"
