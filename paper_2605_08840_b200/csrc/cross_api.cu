// C ABI of the cross attention: argument checks and the choice of the kernel.
#include <cmath>

#include "cross.cuh"
#include "restkv_handle.cuh"

namespace restkv {

static restkv_status make_cross(const restkv_cross* s, int n_tokens, CrossProblem* out) {
  if (!s) return RESTKV_ERR_INVALID_ARG;
  if (s->sources < 1 || s->beams < 1 || s->n_q_heads < 1 || s->n_kv_heads < 1 || s->head_dim < 1 || s->n_rows < 1 || n_tokens < 1) return RESTKV_ERR_INVALID_ARG;
  if (s->n_q_heads % s->n_kv_heads != 0) return RESTKV_ERR_INVALID_ARG;
  if (s->dtype != RESTKV_BF16 && s->dtype != RESTKV_F32) return RESTKV_ERR_INVALID_ARG;
  if (s->lengths_per_head != 0 && s->lengths_per_head != 1) return RESTKV_ERR_INVALID_ARG;
  CrossProblem c{};
  c.sources = s->sources; c.beams = s->beams; c.Hq = s->n_q_heads; c.Hkv = s->n_kv_heads; c.G = c.Hq / c.Hkv; c.d = s->head_dim;
  c.n_rows = s->n_rows; c.per_head = s->lengths_per_head; c.n_tokens = n_tokens;
  c.scale = s->softmax_scale != 0.f ? s->softmax_scale : 1.0f / sqrtf((float)c.d);
  if (!(c.scale > 0.f) || !std::isfinite(c.scale)) return RESTKV_ERR_INVALID_ARG;
  if (c.d % 8 != 0 || c.d > 256) return RESTKV_ERR_UNSUPPORTED;
  if (c.n_rows > 0x7FFFFFFF - 256) return RESTKV_ERR_UNSUPPORTED;                      // rows, rounded up to tiles, are counted in 32 bits
  if ((long long)c.sources * c.Hkv > 65535) return RESTKV_ERR_UNSUPPORTED;             // a grid's third dimension
  if ((long long)c.sources * c.beams > 0x7FFFFFFFll) return RESTKV_ERR_UNSUPPORTED;
  // query rows of a KV head, rounded up to tiles, too
  if ((long long)c.beams * n_tokens > 0x7FFFFFFFll || (long long)c.beams * n_tokens > (0x7FFFFFFFll - 256) / c.G) return RESTKV_ERR_UNSUPPORTED;
  *out = c;
  return RESTKV_OK;
}

// Rows [batch, heads, n, d]; the strides of dimensions of extent 1 are nobody's business.
static restkv_status make_view(const restkv_rows* s, int batch, int heads, int n, int d, RowsView* out) {
  if (!s || !s->data || !aligned16(s->data)) return RESTKV_ERR_INVALID_ARG;
  RowsView v{s->data, s->stride_b, s->stride_h, s->stride_n};
  if (v.sb == 0 && v.sh == 0 && v.sn == 0) v = RowsView{s->data, (long long)heads * n * d, (long long)n * d, d};
  if (n == 1) v.sn = d;
  if (heads == 1) v.sh = (long long)n * d;
  if (batch == 1) v.sb = (long long)heads * n * d;
  for (long long st : {v.sb, v.sh, v.sn})
    if (st < 0 || st % 8 != 0) return RESTKV_ERR_INVALID_ARG;
  *out = v;
  return RESTKV_OK;
}

// The most that any kernel that the call can run on needs.  It never falls as n_tokens grows (each part rises with them and, once there, stays).
static size_t cross_bytes(const CrossProblem& c, bool f32, int sm_count) {
  size_t most = cross_simt_bytes(c, sm_count);
  if (!f32 && cross_few_bytes(c, sm_count) > most) most = cross_few_bytes(c, sm_count);
  if (!f32 && cross_many_bytes(c, sm_count) > most) most = cross_many_bytes(c, sm_count);
  return align256(most);
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

size_t restkv_cross_workspace_bytes(const restkv_cross* cross, int n_tokens) {
  CrossProblem c;
  if (make_cross(cross, n_tokens, &c) != RESTKV_OK) return 0;
  return cross_bytes(c, cross->dtype == RESTKV_F32, current_sms());
}

restkv_status restkv_cross_attend(restkv_handle* h, const restkv_cross* cross, int n_tokens, const restkv_rows* Q, const restkv_rows* K,
                                  const restkv_rows* V, const int32_t* lengths, const int32_t* counts, void* out, float* lse, void* workspace,
                                  size_t workspace_bytes, restkv_stream stream) {
  if (!h || !out || !aligned16(out)) return RESTKV_ERR_INVALID_ARG;
  CrossProblem c;
  restkv_status s = make_cross(cross, n_tokens, &c);
  if (s != RESTKV_OK) return s;
  if (c.per_head && !lengths) return RESTKV_ERR_INVALID_ARG;
  if ((s = make_view(Q, c.sources * c.beams, c.Hq, n_tokens, c.d, &c.Q)) != RESTKV_OK) return s;
  if ((s = make_view(K, c.sources, c.Hkv, c.n_rows, c.d, &c.K)) != RESTKV_OK) return s;
  if ((s = make_view(V, c.sources, c.Hkv, c.n_rows, c.d, &c.V)) != RESTKV_OK) return s;
  const bool f32 = cross->dtype == RESTKV_F32;
  if (!workspace || ((uintptr_t)workspace & 255u) != 0 || workspace_bytes < cross_bytes(c, f32, h->sm_count)) return RESTKV_ERR_WORKSPACE;
  if (!on_device(h)) return RESTKV_ERR_INVALID_ARG;
  c.lengths = lengths; c.counts = counts; c.out = out; c.lse = lse;
  Call call{h, (cudaStream_t)stream};
  const bool tensor_cores = !f32 && h->tc_state && h->kernel_path != 1;
  const bool few = h->cross_few && cross_few_supported(c), many = h->cross_many && cross_many_supported(c);
  if (tensor_cores && many && (!few || cross_many_us(c, h->sm_count) < cross_few_us(c, h->paged_clusters[0]))) {
    RESTKV_LAUNCH(call, RESTKV_KERNEL_NONE, launch_cross_many(h->tc_state, c, (float*)workspace, h->sm_count, h->wait_limit, h->dev_status, call.st), 2);
    return RESTKV_OK;
  }
  if (tensor_cores && few) {
    int launches = 0;
    RESTKV_LAUNCH(call, RESTKV_KERNEL_NONE,
                  launch_cross_few(h->tc_state, c, (float*)workspace, h->sm_count, h->paged_clusters[0], h->wait_limit, h->dev_status, call.st, &launches), launches);
    return RESTKV_OK;
  }
  if (h->kernel_path >= 2) return RESTKV_ERR_UNSUPPORTED;   // the tensor cores are required
  const int splits = cross_simt_splits(c, h->sm_count);
  RESTKV_LAUNCH(call, RESTKV_KERNEL_NONE, launch_cross_simt(c, f32, (float*)workspace, splits, call.st), splits == 1 ? 1 : 2);
  return RESTKV_OK;
}

}  // extern "C"
